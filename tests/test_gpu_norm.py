"""The RMS norm against its 64-bit form: rows of every width, both storage types, the residual's sum in place and apart, 8-bit
outputs bit by bit, gradients."""
import numpy as np
import pytest
import torch

import block_ref
import paper_2503_01868_amd as hy

from gpu_util import say

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
WIDTHS = [1, 7, 64, 100, 512, 513, 1000, 1024, 1025, 2048, 2050, 4096, 8192, 8200, 16384, 20000, 16388, 2500, 5003]


def make(seed, shape, dtype, scale=1.0):
    rng = np.random.default_rng(seed)
    return torch.from_numpy((rng.normal(size=shape) * scale).astype(np.float32)).to(DTYPES[dtype]).cuda()


def wide(t):
    return t.double().cpu().numpy()


def close(got, ref, size, dtype, what):
    """fp32 arithmetic: 1e-5 of the terms' magnitudes (a sum in pieces of some 100 roundings of 6e-8); a stored bf16 element besides:
    2^-8 of itself."""
    got = wide(got)
    assert got.shape == ref.shape, what
    assert np.isfinite(got).all(), what
    worst = np.abs(got - ref) - 1e-5 * size - (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0.0)
    assert not worst.size or worst.max() <= 1e-30, (what, worst.max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", WIDTHS)
def test_forward_and_gradients(D, dtype):
    for N, residual, weights in ((5, True, True), (1, False, False), (700 if D <= 1100 else 9, True, True)):
        say("norm N=%d D=%d %s" % (N, D, dtype))
        x, dy, dh = (make(D + i, (N, D), dtype) for i in range(3))
        r = make(D + 3, (N, D), dtype, 2.0) if residual else None
        w = make(D + 4, (D,), dtype) if weights else None
        y, total, rstd = hy.hyena_rmsnorm_fwd(x, w, residual=r, eps=1e-5, want_rstd=True)
        if residual:
            assert torch.equal(total, (x.float() + r.float()).to(x.dtype))
        else:
            assert total is x
        h, w64 = wide(total), None if w is None else wide(w)
        ry, _, rr = block_ref.rmsnorm(h, w64, eps=1e-5)
        close(y, ry, np.abs(ry), dtype, "y")
        close(rstd, rr, rr, "f32", "rstd")
        dx, dw = hy.hyena_rmsnorm_bwd(dy, total, rstd, w, dtotal=dh if residual else None)
        rx, rw = block_ref.rmsnorm_grads(wide(dy), h, w64, wide(dh) if residual else None, eps=1e-5)
        # (the magnitudes of what is subtracted: every term of the inner sum)
        wdy = np.abs(wide(dy)) * (1.0 if w is None else np.abs(w64))
        size = rr[:, None] * (wdy + np.abs(h) * rr[:, None] ** 2 * (wdy * np.abs(h)).mean(1, keepdims=True)) + np.abs(wide(dh))
        close(dx, rx, size, dtype, "dx")
        if weights:
            close(dw, rw, (np.abs(wide(dy) * h) * rr[:, None]).sum(0), dtype, "dw")
            assert torch.equal(hy.hyena_rmsnorm_bwd(dy, total, rstd, w, dtotal=dh if residual else None)[1], dw)
            assert hy.hyena_rmsnorm_bwd(dy, total, rstd, w, want_dw=False)[1] is None
        else:
            assert dw is None


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [1, 7, 64, 1000, 1032, 4096, 5003, 8192, 20000])
def test_eight_bits_bit_by_bit(D, dtype):
    """The numbers depend on products of two inputs and one quotient alone, each rounded to fp32."""
    N = 6
    x, r, w = make(D, (N, D), dtype), make(D + 1, (N, D), dtype, 3.0), make(D + 2, (D,), dtype)
    x[2], r[2] = 0, 0
    x[3] *= 2.0 ** -60
    r[3] = 0
    x[4, 0] = 1e4
    for weights, residual in ((w, r), (None, None)):
        y, scale, total, rstd = hy.hyena_rmsnorm_fwd_8bit(x, weights, residual=residual, want_rstd=True)
        assert y.dtype == torch.float8_e4m3fn
        u = total.float().cpu() if weights is None else total.float().cpu() * w.float().cpu()
        top = u.abs().amax(1, keepdim=True)
        some = top >= 2.0 ** -100
        want = (u * torch.where(some, torch.full_like(top, 448.0) / top, 0.0)).to(torch.float8_e4m3fn)
        assert torch.equal(y.cpu().view(torch.uint8), want.view(torch.uint8))
        ry, _, rr = block_ref.rmsnorm(wide(total), None if weights is None else wide(w))
        close(scale, wide(top)[:, 0] / 448 * rr, wide(top)[:, 0] / 448 * rr, "f32", "scale")
        close(rstd, rr, rr, "f32", "rstd")
        value = wide(y.float()) * wide(scale)[:, None]
        assert np.abs(value - ry).max() <= np.abs(ry).max() * (2.0 ** -4 + 1e-5)


def test_eight_bits_of_what_is_not_finite():
    x = make(1, (4, 64), "bf16")
    x[0, 3], x[1, 5] = float("inf"), float("nan")
    y, scale, _, _ = hy.hyena_rmsnorm_fwd_8bit(x)
    value = y.float() * scale[:, None]
    assert torch.isnan(value[0, 3]) and (value[0, :3] == 0).all() and (value[0, 4:] == 0).all()
    assert torch.isnan(value[1]).all() and torch.isfinite(value[2:]).all()
    assert torch.isfinite(y.float()[1, :5]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [7, 1000, 4096, 20000])
def test_in_place(D, dtype):
    """The sum in the residual's or x's own place; the gradient in that of what comes back along the residual, or of dy."""
    N = 5
    x, r, w, dy, dh = (make(D + i, s, dtype) for i, s in enumerate([(N, D), (N, D), (D,), (N, D), (N, D)]))
    y, total, rstd = hy.hyena_rmsnorm_fwd(x, w, residual=r, want_rstd=True)
    for own in ("residual", "x"):
        cx, cr = x.clone(), r.clone()
        z, t, _ = hy.hyena_rmsnorm_fwd(cx, w, residual=cr, total=cr if own == "residual" else cx)
        assert torch.equal(z, y) and torch.equal(t, total) and t is (cr if own == "residual" else cx)
        assert torch.equal(cx if own == "residual" else cr, x if own == "residual" else r)
    dx, dw = hy.hyena_rmsnorm_bwd(dy, total, rstd, w, dtotal=dh)
    for own in ("dtotal", "dy"):
        cdy, cdh = dy.clone(), dh.clone()
        z, v = hy.hyena_rmsnorm_bwd(cdy, total, rstd, w, dtotal=cdh, dx=cdh if own == "dtotal" else cdy)
        assert torch.equal(z, dx) and torch.equal(v, dw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views_broadcasts_and_odd_places(dtype):
    N, D = 12, 64
    x, r, w = make(1, (N, D), dtype), make(2, (N, D), dtype), make(3, (D,), dtype)
    y, total, _ = hy.hyena_rmsnorm_fwd(x, w, residual=r)
    fused = torch.cat([x, r], 1)
    z, t, _ = hy.hyena_rmsnorm_fwd(fused[:, :D], w, residual=fused[:, D:])
    assert torch.equal(z, y) and torch.equal(t, total)
    odd = torch.empty(N * D + 1, dtype=x.dtype, device="cuda")[1:].view(N, D).copy_(x)
    assert (hy.hyena_rmsnorm_fwd(odd, w, residual=r)[0] - y).abs().max() <= 2.0 ** -7 * y.abs().max()
    same = r[:1].expand(N, D)
    z, t, _ = hy.hyena_rmsnorm_fwd(x, w, residual=same)
    assert torch.equal(t, (x.float() + same.float()).to(x.dtype))
    z, t, rstd = hy.hyena_rmsnorm_fwd(x.view(3, 4, D), w, residual=r.view(3, 4, D), want_rstd=True)
    assert z.shape == (3, 4, D) and rstd.shape == (3, 4) and torch.equal(z.view(N, D), y)
    three = fused.view(3, 4, 2 * D)[..., :D]
    assert torch.equal(hy.hyena_rmsnorm_fwd(three, w, residual=r.view(3, 4, D))[0].view(N, D), y)


def test_rows_of_zeros_and_no_rows():
    x = torch.zeros(3, 128, device="cuda")
    y, _, rstd = hy.hyena_rmsnorm_fwd(x, want_rstd=True, eps=1e-4)
    assert (y == 0).all() and torch.allclose(rstd, torch.full_like(rstd, 100.0), rtol=1e-6)
    w = torch.ones(128, device="cuda")
    empty = x[:0]
    y, total, rstd = hy.hyena_rmsnorm_fwd(empty, w, residual=empty, want_rstd=True)
    assert y.shape == empty.shape and rstd.shape == (0,)
    dx, dw = hy.hyena_rmsnorm_bwd(empty, total, rstd, w)
    assert dx.shape == empty.shape and (dw == 0).all()


def test_outputs_end_where_they_end():
    for D in (7, 64, 1000):
        x = make(1, (5, D), "bf16")
        guard = torch.full((5 * D + 64,), 3.0, dtype=x.dtype, device="cuda")
        hy.hyena_rmsnorm_fwd(x, out=guard[:5 * D].view(5, D))
        assert (guard[5 * D:] == 3).all()


def test_refusals():
    x, w = make(1, (4, 64), "bf16"), make(2, (64,), "bf16")
    for bad in (dict(w=w.float()), dict(w=w[:32]), dict(residual=x[:2]), dict(residual=x.float()), dict(x=x.t()), dict(x=x.cpu()), dict(total=x.clone()),
                dict(residual=x, total=x[:2]), dict(x=make(1, (4, 8, 4, 64), "bf16").transpose(0, 1))):
        with pytest.raises(ValueError):
            hy.hyena_rmsnorm_fwd(**{**dict(x=x, w=w), **bad})
    with pytest.raises(hy.HyenaError):   # in place on rows that are further apart
        both = torch.cat([x, x], 1)
        hy.hyena_rmsnorm_fwd(x, w, residual=both[:, :64], total=both.view(-1)[:4 * 64].view(4, 64))
    with pytest.raises(hy.HyenaError):
        hy.hyena_rmsnorm_fwd(x, w, eps=-1.0)
    with pytest.raises(TypeError):
        hy.hyena_rmsnorm_fwd(x.half())
    _, total, rstd = hy.hyena_rmsnorm_fwd(x, w, want_rstd=True)
    with pytest.raises(ValueError):
        hy.hyena_rmsnorm_bwd(x, total, rstd.half(), w)
    with pytest.raises(ValueError):
        hy.hyena_rmsnorm_bwd(x, total[:2], rstd, w)
