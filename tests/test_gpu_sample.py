"""The choice of tokens against its 64-bit form: every limit alone and together, ties, borders, what is not finite, vocabularies from
one word to a million."""
import math

import numpy as np
import pytest
import torch

import block_ref
import paper_2503_01868_amd as hy

from gpu_util import say

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def check(z, u, temperature=1.0, top_k=None, top_p=None, min_p=None):
    """Tokens equal; the probability is rounded to fp32 once, and its sums are in double."""
    token, prob = hy.hyena_sample(z, u, temperature, top_k, top_p, min_p)

    def one(x, n, otherwise):
        return otherwise if x is None else float(x[n]) if isinstance(x, torch.Tensor) else x

    rows, us = z.double().cpu().numpy(), u.double().cpu().numpy()
    for n in range(z.shape[0]):
        want, p = block_ref.sample(rows[n], us[n], one(temperature, n, 1.0), int(one(top_k, n, 0)), one(top_p, n, 1.0), one(min_p, n, 0.0))
        assert int(token[n]) == want, (n, int(token[n]), want)
        assert abs(float(prob[n]) - p) <= 2.0 ** -23 * p, n


def make(seed, N, V, dtype, scale=2.5):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy((rng.normal(size=(N, V)) * scale).astype(np.float32)).to(DTYPES[dtype]).cuda()
    return z, torch.from_numpy(rng.uniform(size=N).astype(np.float32)).cuda(), rng


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 7, 63, 64, 65, 511, 512, 513, 2048, 2049, 5003, 32768, 40001])
def test_every_limit_alone_and_together(V, dtype):
    N = 5
    z, u, rng = make(V, N, V, dtype)
    t = torch.from_numpy(rng.uniform(0.5, 1.5, size=N).astype(np.float32)).cuda()
    k = torch.from_numpy(rng.integers(1, max(2, min(V, 300)), size=N).astype(np.int32)).cuda()
    p = torch.from_numpy(rng.uniform(0.2, 1, size=N).astype(np.float32)).cuda()
    m = torch.from_numpy(rng.uniform(1e-3, 0.2, size=N).astype(np.float32)).cuda()
    say("sample V=%d %s" % (V, dtype))
    check(z, u)
    check(z, u, t)
    check(z, u, t, top_k=k)
    check(z, u, t, top_p=p)
    check(z, u, t, min_p=m)
    check(z, u, t, k, p, m)
    check(z, u, 0.7, 20, 0.9, 0.05)
    check(z, u, 0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_go_to_the_lowest_index(dtype):
    """Few different logits: every border of top-k and top-p falls among equal ones."""
    N, V = 40, 3001
    rng = np.random.default_rng(3)
    z = torch.from_numpy(rng.integers(-3, 3, size=(N, V)).astype(np.float32)).to(DTYPES[dtype]).cuda()
    u = torch.from_numpy(rng.uniform(size=N).astype(np.float32)).cuda()
    k = torch.from_numpy(rng.integers(1, V, size=N).astype(np.int32)).cuda()
    p = torch.from_numpy(rng.uniform(size=N).astype(np.float32)).cuda()
    check(z, u, 1.0, top_k=k)
    check(z, u, 1.0, top_p=p)
    check(z, u, 1.3, k, p)
    check(z, u, 0.0)
    flat = torch.zeros_like(z)
    check(flat, u)
    check(flat, u, 1.0, k, p)
    assert (hy.hyena_sample(flat, u, 0.0)[0] == 0).all()
    signs = torch.tensor([[-0.0, 0.0, -0.0, -1.0]], dtype=z.dtype, device="cuda")  # equal, all three zeros
    assert int(hy.hyena_sample(signs, u[:1], 0.0)[0]) == 0
    assert int(hy.hyena_sample(signs, torch.full_like(u[:1], 0.99), 1.0, top_k=2)[0]) == 1


def test_exact_borders():
    """Powers of two: sums and products are exact, so the border itself is defined: a sum has to pass u, and to reach top_p."""
    z = torch.tensor([[0.0, -1.0, -2.0, -2.0]], device="cuda") * math.log(2.0)
    z = torch.tensor([[0.0, 0.0, 0.0, 0.0]], device="cuda").expand(8, 4)
    u = torch.tensor([0.0, 0.2499, 0.25, 0.4999, 0.5, 0.75, 0.9999, 1.0], device="cuda")
    token, prob = hy.hyena_sample(z, u)
    assert token.tolist() == [0, 0, 1, 1, 2, 3, 3, 3] and (prob == 0.25).all()
    for p, kept in ((0.25, 1), (0.2501, 2), (0.5, 2), (0.75, 3), (0.7501, 4), (0.0, 1), (-1.0, 1), (1.0, 4), (float("nan"), 4)):
        token, prob = hy.hyena_sample(z[:1], torch.tensor([0.9999], device="cuda"), top_p=torch.tensor([p], device="cuda"))
        assert int(token) == kept - 1 and float(prob) == np.float32(1 / kept), p
    assert int(hy.hyena_sample(z[:1], torch.tensor([0.9999], device="cuda"), min_p=1.0)[0]) == 3


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_finite(dtype):
    inf, nan = float("inf"), float("nan")
    z, _, rng = make(4, 8, 700, dtype)
    u = torch.from_numpy(rng.uniform(size=8).astype(np.float32)).cuda()
    z[0] = -inf
    z[1, 1:] = -inf
    z[2, ::2] = nan
    z[3, 5], z[3, 600] = inf, inf
    z[4, :] = nan
    z[5, :699] = -inf
    z[6, 10] = 3e38 if dtype == "f32" else 3e38
    for t in (1.0, 0.0, 1e-30):
        check(z, u, t)
        check(z, u, t, 3, 0.9, 0.1)
        check(z, u, t, 650, 0.999999)
    token, prob = hy.hyena_sample(z, u)
    assert token[0] == -1 and prob[0] == 0 and token[4] == -1 and token[1] == 0 and token[5] == 699
    z = torch.zeros(1, 8, dtype=z.dtype, device="cuda")
    for bad in (nan, -1.0):
        assert int(hy.hyena_sample(z, torch.tensor([bad], device="cuda"))[0]) == 0
    assert int(hy.hyena_sample(z, torch.tensor([0.9], device="cuda"), torch.tensor([nan], device="cuda"), min_p=torch.tensor([nan], device="cuda"))[0]) == 7


def test_a_u_of_zero_takes_the_first_word_that_has_any_weight():
    z = torch.tensor([[-60.0, -300.0, 0.0, 1.0], [-2000.0, -60.0, 1.0, 0.0]], device="cuda")
    assert hy.hyena_sample(z, torch.zeros(2, device="cuda"))[0].tolist() == [0, 1]


@pytest.mark.parametrize("dtype,V", [("bf16", 65536), ("f32", 131072), ("f32", 1 << 20), ("bf16", (1 << 20) + 7)])
def test_large_vocabularies(dtype, V):
    """Against the same in torch's double on the GPU: sorted, summed in order."""
    N = 6
    z, u, rng = make(7, N, V, dtype)
    t = torch.from_numpy(rng.uniform(0.5, 1.5, size=N).astype(np.float32)).cuda()
    for k, p, m in ((None, None, None), (50, 0.9, 0.02), (None, 0.95, None), (V // 2, None, None), (None, None, 0.01)):
        token, prob = hy.hyena_sample(z, u, t, k, p, m)
        for n in range(N):
            d = z[n].double()
            w = torch.exp((d - d.max()) / float(t[n]))
            order = torch.sort(d, descending=True, stable=True).indices
            if k is not None:
                order = order[:k]
            if p is not None:
                upto = w[order].cumsum(0)
                order = order[:int((upto < p * upto[-1]).sum()) + 1]
            if m is not None:
                order = order[w[order] >= m]
            words = order.sort().values
            upto = w[words].cumsum(0)
            at = int((upto <= float(u[n]) * upto[-1]).sum())
            assert int(token[n]) == int(words[at]), (n, k, p, m)
            assert abs(float(prob[n]) - float(w[words[at]] / upto[-1])) <= 1e-6 * float(prob[n])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [4096, 4097, 9001, 70001])
def test_what_long_rows_leave_to_choose_from(V, dtype):
    """top_k at the ends of what is gathered from a row, words in a few runs, among infinities and NaN, rows of equal logits, rows
    that begin anywhere."""
    N = 4
    z, u, rng = make(V + 1, N, V, dtype)
    say("sample long V=%d %s" % (V, dtype))
    for k in (1, 2, 1000, 2047, 2048, 2049, 4095):
        check(z, u, 1.1, top_k=k)
        check(z, u, 0.9, k, 0.9, 0.01)
    for m in (1e-300, 1e-4, 0.3, 1.0, 2.0):
        check(z, u, 1.3, min_p=m)
    crowded = z.clone()
    crowded[0, :3000] += 20  # what counts lies in the first pieces
    crowded[1, V // 2:V // 2 + 50] += 20
    crowded[2] = 1.0
    crowded[3] = -float("inf")
    crowded[3, [5, V - 1]] = 0.0
    check(crowded, u, 1.0, 40, 0.95, 0.01)
    check(crowded, u, 1.0, min_p=0.5)
    check(crowded, u, 1.0, 2000, 0.5)
    odd = z.clone()
    odd[0, ::3] = float("nan")
    odd[1, [7, V // 2, V - 2]] = float("inf")
    odd[2, ::2] = -float("inf")
    odd[3] = -odd[3].abs()
    for t in (1.0, 1e-30, float("inf")):
        check(odd, u, t, 50, 0.9)
        check(odd, u, t, min_p=0.1)
    check(odd, u, 0.0)
    few = torch.from_numpy(rng.integers(-20, 3, size=(N, V)).astype(np.float32)).to(DTYPES[dtype]).cuda()
    few[:, 1000:] -= 40
    check(few, u, 1.0, 60, 0.7)
    for first in (1, 2, 3, 5):
        padded = torch.full((N, V + 9), float("nan"), dtype=z.dtype, device="cuda")
        padded[:, first:V + first] = z
        check(padded[:, first:V + first], u, 0.8, 30, 0.9)
        check(padded[:, first:V + first], u, 0.8)
        check(padded[:, first:V + first], u, 0.0)


def test_tokens_come_as_often_as_they_are_likely():
    z, _, _ = make(8, 1, 300, "f32")
    N = 20000
    u = (torch.arange(N, device="cuda") + 0.5) / N
    token, prob = hy.hyena_sample(z.expand(N, 300), u, 0.9)
    p = torch.softmax(z.double()[0] / 0.9, 0)
    assert (torch.bincount(token, minlength=300) / N - p).abs().max() <= 1.5 / N
    assert (prob.double() - p[token]).abs().max() <= 1e-7


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views(dtype):
    z, u, _ = make(9, 6, 1001, dtype)
    want = hy.hyena_sample(z, u, 0.8, 30, 0.9)[0]
    padded = torch.full((6, 1100), float("nan"), dtype=z.dtype, device="cuda")
    padded[:, 3:1004] = z
    assert torch.equal(hy.hyena_sample(padded[:, 3:1004], u, 0.8, 30, 0.9)[0], want)
    assert torch.equal(hy.hyena_sample(z[::2], u[::2].contiguous(), 0.8, 30, 0.9)[0], want[::2])
    token, prob = hy.hyena_sample(z, u, want_prob=False)
    assert prob is None
    assert hy.hyena_sample(z[:0], u[:0])[0].shape == (0,)


def test_refusals():
    z, u, _ = make(10, 4, 100, "f32")
    for bad in (dict(u=u[:2]), dict(u=u.double()), dict(logits=z.t()), dict(logits=z[:, :0]), dict(logits=z[0]), dict(top_k=u), dict(logits=z.cpu()),
                dict(temperature=u[:1]), dict(top_p=u.double()), dict(min_p=u.cpu())):
        with pytest.raises(ValueError):
            hy.hyena_sample(**{**dict(logits=z, u=u), **bad})
    with pytest.raises(TypeError):
        hy.hyena_sample(z.half(), u)
