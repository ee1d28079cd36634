"""The natively marshalled calls of the norm, the single token and the choice of tokens: the same bits as the binding's own path, and that
path for whatever is not plain."""
import pytest
import torch

import paper_2503_01868_amd as hy
from paper_2503_01868_amd import binding

from gpu_util import say

pytestmark = pytest.mark.gpu


def normal(seed, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator(device="cuda:0").manual_seed(seed), device="cuda:0").to(dtype)


def calls(dtype):
    x, r, dy = (normal(i, 2, 9, 200, dtype=dtype) for i in range(3))
    w = normal(3, 200, dtype=dtype)
    _, total, rstd = hy.hyena_rmsnorm_fwd(x, w, residual=r, want_rstd=True)
    q, k, v, g = normal(4, 3, 2, 40, dtype=dtype), normal(5, 3, 2, 40, dtype=dtype), normal(6, 3, 6, 72, dtype=dtype), -normal(7, 3, 6, dtype=dtype).abs()
    z, u = normal(8, 5, 3000, dtype=dtype), torch.rand(5, device="cuda:0")
    top_k = torch.arange(1, 6, device="cuda:0", dtype=torch.int32)
    t, p, m = u + 0.5, 1 - u / 2, u / 20

    def step(*args):
        state = normal(9, 3, 6, 40, 72)
        return hy.hyena_la_step(*args[:4], state, *args[4:]), state

    return [("norm", lambda: hy.hyena_rmsnorm_fwd(x, w, residual=r, want_rstd=True)), ("norm alone", lambda: hy.hyena_rmsnorm_fwd(x)),
            ("norm in 8 bits", lambda: hy.hyena_rmsnorm_fwd_8bit(x, w, residual=r, want_rstd=True)),
            ("norm alone in 8 bits", lambda: hy.hyena_rmsnorm_fwd_8bit(x)),
            ("norm bwd", lambda: hy.hyena_rmsnorm_bwd(dy, total, rstd, w, dtotal=r)), ("norm bwd alone", lambda: hy.hyena_rmsnorm_bwd(dy, total, rstd)),
            ("norm bwd without dw", lambda: hy.hyena_rmsnorm_bwd(dy, total, rstd, w, want_dw=False)), ("step", lambda: step(q, k, v, g, 0.3)),
            ("sample", lambda: hy.hyena_sample(z, u, t, top_k, p, m)), ("sample by numbers", lambda: hy.hyena_sample(z, u, 0.7, 20, 0.9, 0.01)),
            ("sample by whole numbers", lambda: hy.hyena_sample(z, u, 1, 20, 1, 0)), ("sample plainly", lambda: hy.hyena_sample(z, u)),
            ("greedy", lambda: hy.hyena_sample(z, u, 0.0))]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_the_same_bits(dtype, monkeypatch):
    binding.lib()
    assert binding._fast is not binding._Unmarshalled
    made = calls(dtype)
    stream = torch.cuda.Stream()
    for name, call in made:
        say("marshalled %s %s" % (name, dtype))
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            fast = call()
        stream.synchronize()
        with monkeypatch.context() as m:
            m.setattr(binding, "_fast", binding._Unmarshalled)
            slow = call()
        torch.cuda.synchronize()
        assert isinstance(fast, tuple) and len(fast) == len(slow)
        for x, y in zip(fast, slow):
            assert (x is None) == (y is None), name
            if x is not None and x.dtype == torch.float8_e4m3fn:
                x, y = x.view(torch.uint8), y.view(torch.uint8)
            assert x is None or (torch.equal(x, y) and x.dtype == y.dtype and not x.requires_grad), name
    x = normal(1, 4, 64, dtype=dtype)
    assert hy.hyena_rmsnorm_fwd(x)[1] is x


def test_what_is_not_plain_takes_the_other_path():
    x, w = normal(1, 8, 64), normal(2, 64)
    binding.lib()
    fast = binding._fast
    for bad in ((x[:, ::2], None, None, 1e-6, False), (x, w.double(), None, 1e-6, False), (x, w[:32], None, 1e-6, False), (x, w, x[:4], 1e-6, False),
                (x.cpu(), None, None, 1e-6, False), (x.half(), None, None, 1e-6, False), (None, None, None, 1e-6, False), (x, w, None, "1", False),
                (x[:0], w, None, 1e-6, False)):
        assert fast.norm_fwd(*bad, False) is None and fast.norm_fwd(*bad, True) is None
    rstd = torch.ones(8, device="cuda:0")
    for bad in ((x, None, rstd, w, None, True), (x, x, None, w, None, True), (x, x, rstd[:4], w, None, True), (x, x, rstd, w[:3], None, True),
                (x, x, rstd.bfloat16(), w, None, True), (x, x, rstd, w, x[:1], True), (x, x.bfloat16(), rstd, w, None, True)):
        assert fast.norm_bwd(*bad) is None
    q, v, g, state = normal(3, 2, 2, 8), normal(4, 2, 4, 8), normal(5, 2, 4), normal(6, 2, 4, 8, 8)
    for bad in ((q, q, v, g, state[:1], 1.0), (q, q[:1], v, g, state, 1.0), (q, q, v[:, :3], g, state, 1.0), (q, q, v, g[:, :2], state, 1.0),
                (q, q, v, g, state.bfloat16(), 1.0), (q, q, v, g, None, 1.0), (q, q, v, g, state, None), (q, q, v.bfloat16(), g, state, 1.0)):
        assert fast.la_step(*bad) is None
    z, u = normal(7, 4, 50), torch.rand(4, device="cuda:0")
    for bad in ((z, u[:2], 1.0, None, None, None), (z, u.double(), 1.0, None, None, None), (z.t(), u, 1.0, None, None, None), (z, u, u[:1], None, None, None),
                (z, u, 1.0, u, None, None), (z, u, 1.0, 2.5, None, None), (z, u, 1.0, 2 ** 40, None, None), (z[:0], u[:0], 1.0, None, None, None),
                (z, None, 1.0, None, None, None)):
        assert fast.sample(*bad) is None
    assert hy.hyena_sample(z, u, 1.0, top_k=2 ** 40)[0].shape == (4,)
    with pytest.raises(ValueError):
        hy.hyena_rmsnorm_fwd(x, w[:32])
