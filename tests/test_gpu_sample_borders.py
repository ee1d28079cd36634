"""The borders of the choice of tokens: the word that a limit stops at is that of the definition in 64 bits, in every way that a row
is taken (a list of all words, a list gathered from a long row, a long row digit by digit)."""
import math

import numpy as np
import pytest
import torch

import block_ref
import paper_2503_01868_amd as hy

from gpu_util import say

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def falling(V, dtype):
    """One likely word and a tail of unlikely ones, the likelier first: the last word that is kept has the highest index."""
    z = np.concatenate([[0.0], np.linspace(-13.0, -15.0, V - 1)]) if V > 1 else np.zeros(1)
    return torch.from_numpy(z.astype(np.float32)).to(DTYPES[dtype]).cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,top_k", [(1, 1000, None), (1, 4096, None), (1, 9001, 2000), (2, 9001, None), (2, 131072, None), (2, 131072, 100000),
                                       (300, 2048, None), (300, 20001, None)])
def test_top_p_stops_at_the_word_that_reaches_it(N, V, top_k, dtype):
    """top_p next to a sum of weights on both sides, 3e-13 of it away.  The kernel's weights are off by 3 x 2^-53 of themselves for each
    unit of their exponent, 15 x 3 x 1.2e-16 = 5e-15, and its sums by V 2^-62, 3e-14 at most."""
    say("sample top_p N=%d V=%d %s" % (N, V, dtype))
    row = falling(V, dtype)
    kept = V if top_k is None else top_k
    w = np.exp(row.double().cpu().numpy()[:kept]).astype(np.longdouble)
    upto = np.cumsum(w)
    z, u = row.expand(N, V), torch.ones(N, device="cuda")  # (u of 1: the last word that is kept)
    for k in sorted({1, 2, 17, kept // 3, kept // 2, (2 * kept) // 3, kept - 2}):
        p = float(upto[k - 1] / upto[-1])
        for side, last in ((1 - 3e-13, k - 1), (1 + 3e-13, k)):
            token, prob = hy.hyena_sample(z, u, 1.0, top_k, p * side)
            assert token.tolist() == [last] * N, (k, side)
            want = float(w[last] / upto[last])
            assert (prob.double() - want).abs().max() <= 2.0 ** -23 * want


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V", [(3, 700), (3, 9001), (260, 2500)])
def test_min_p_keeps_words_whose_weight_rounds_to_it(N, V, dtype):
    """Weights that are 1 in 64 bits though their logits are below the largest: by a temperature that leaves nothing of the distance, or
    logits next to each other."""
    say("sample min_p N=%d V=%d %s" % (N, V, dtype))
    rng = np.random.default_rng(V)
    far = torch.from_numpy(rng.normal(size=V).astype(np.float32)).to(DTYPES[dtype]).cuda()
    far[5] = -math.inf
    near = torch.from_numpy(rng.choice([0.0, -1e-17, -3e-20, -1.0], size=V).astype(np.float32)).to(DTYPES[dtype]).cuda()
    us = torch.from_numpy(rng.uniform(size=N).astype(np.float32)).cuda()
    for z, t in ((far, 1e20), (far, math.inf), (near, 1.0)):
        token, prob = hy.hyena_sample(z.expand(N, V), us, t, min_p=1.0)
        row = z.double().cpu().numpy()
        for n in range(min(N, 3)):
            want, p = block_ref.sample(row, float(us[n]), t, min_p=1.0)
            assert int(token[n]) == want and abs(float(prob[n]) - p) <= 2.0 ** -23 * p, (t, n)


@pytest.mark.parametrize("N,V", [(64, 700), (64, 4000), (64, 9001), (8, 131072), (300, 2000), (300, 20001)])
@pytest.mark.parametrize("top_k", [None, 300])
def test_a_u_of_one_takes_the_last_word_that_is_kept(top_k, N, V):
    """Whatever the sums round to: of rows whose last words are all unlikely."""
    say("sample u = 1 N=%d V=%d" % (N, V))
    z = torch.randn(N, V, generator=torch.Generator(device="cuda").manual_seed(V), device="cuda") * 2.5
    if top_k is None:
        z[:, -3:] = -60.0
        last = torch.full((N,), V - 1, device="cuda")
    else:
        last = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :top_k].amax(1)
    for u in (1.0, 2.0, math.inf):
        assert torch.equal(hy.hyena_sample(z, torch.full((N,), u, device="cuda"), 1.0, top_k)[0], last), u


@pytest.mark.parametrize("N,V", [(3, 700), (3, 9001), (260, 2500)])
def test_weights_below_the_smallest_normal_number_are_weights(N, V):
    """exp(-744) is 1e-323 in 64 bits: a u of zero takes the first word that has any weight, and a u of one the last."""
    say("sample smallest weights N=%d V=%d" % (N, V))
    z = torch.linspace(-50.0, 0.0, V, device="cuda")
    for far, there in ((-720.0, True), (-744.0, True), (-750.0, False), (-1e5, False)):
        z[0], z[-1] = far, far
        row = z.double().cpu().numpy()
        token, prob = hy.hyena_sample(z.expand(N, V), torch.zeros(N, device="cuda"))
        assert block_ref.sample(row, 0.0)[0] == (0 if there else 1) and (token == (0 if there else 1)).all(), far
        token, prob = hy.hyena_sample(z.expand(N, V), torch.ones(N, device="cuda"))
        assert (token == (V - 1 if there else V - 2)).all(), far


@pytest.mark.parametrize("N,V", [(2, 4), (2, 900), (2, 4096), (2, 9001), (300, 2000), (300, 9001)])
def test_borders_between_unequal_weights(N, V):
    """top_p and min_p 1e-12 beside a border, u at the fp32 numbers on its two sides (a hundredth of their distance away from it at least)."""
    say("sample unequal N=%d V=%d" % (N, V))
    rng = np.random.default_rng(V)
    row = rng.permutation(np.linspace(0.0, -4.0, V)).astype(np.float32)
    z = torch.from_numpy(row).cuda().expand(N, V)
    w = np.exp(row.astype(np.float64) - row.max())
    order = np.argsort(-row, kind="stable")
    one = torch.full((N,), 0.37, device="cuda")
    for k in sorted({1, V // 3, V - 2}):
        upto = np.cumsum(w[order].astype(np.longdouble))
        p, m = float(upto[k - 1] / upto[-1]), float(w[order[k]])
        for kept, limits in ((k, dict(top_p=p * (1 - 1e-12))), (k + 1, dict(top_p=p * (1 + 1e-12))), (k, dict(min_p=m * (1 + 1e-12))),
                             (k + 1, dict(min_p=m * (1 - 1e-12)))):
            # every word that is kept, and none else, in the vocabulary's order: the last of them, and one inside
            words = np.sort(order[:kept])
            sums = np.cumsum(w[words].astype(np.longdouble))
            assert (hy.hyena_sample(z, torch.ones_like(one), 1.0, **limits)[0] == int(words[-1])).all(), (k, limits)
            token, prob = hy.hyena_sample(z, one, 1.0, **limits)
            want = int(words[np.searchsorted(sums, np.float32(0.37) * sums[-1], side="right")])
            assert (token == want).all(), (k, limits)
            p_want = float(w[want] / sums[-1])
            assert (prob.double() - p_want).abs().max() <= 2.0 ** -23 * p_want
    sums = np.cumsum(w.astype(np.longdouble))
    for k in sorted({0, V // 3, V - 2}):
        border = sums[k] / sums[-1]
        below = np.float32(border)
        below = below if below < border else np.nextafter(below, np.float32(0))
        above = np.nextafter(below, np.float32(1))
        gap = float(above) - float(below)
        for x, want in ((below, k), (above, k + 1)):
            if abs(float(x) - float(border)) > gap / 100 and abs(float(x) - float(border)) < float(min(w[k], w[k + 1]) / sums[-1]):
                assert (hy.hyena_sample(z, torch.full((N,), float(x), device="cuda"))[0] == want).all(), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1025, 2049, 9001, 70001])
def test_long_rows_of_more_sequences_than_compute_units(V, dtype):
    """More than 256 rows: other workgroups, lists and borders of lists than few rows have.  Some of the rows against the 64-bit form."""
    N = 257
    say("sample many V=%d %s" % (V, dtype))
    rng = np.random.default_rng(V)
    z = torch.randn(N, V, generator=torch.Generator(device="cuda").manual_seed(V), device="cuda").mul_(2.5).to(DTYPES[dtype])
    z[1, ::3] = math.nan
    z[2, [7, V // 2, V - 2]] = math.inf
    z[3, ::2] = -math.inf
    z[4] = 1.0
    z[5, V // 2:V // 2 + 50] += 20
    z[6] = -math.inf
    z[255] = torch.from_numpy(rng.integers(-3, 3, size=V).astype(np.float32)).to(z.dtype)
    u = torch.from_numpy(rng.uniform(size=N).astype(np.float32)).cuda()
    some = [0, 1, 2, 3, 4, 5, 6, 255, 256] if V < 20000 else [0, 1, 2, 5, 255]
    rows, us = z[some].double().cpu().numpy(), u[some].double().cpu().numpy()

    def check(x, t, top_k=0, top_p=1.0, min_p=0.0):
        token, prob = hy.hyena_sample(x, u, t, top_k, top_p, min_p)
        for i, n in enumerate(some):
            want, p = block_ref.sample(rows[i], us[i], t, top_k, top_p, min_p)
            assert int(token[n]) == want, (n, t, top_k, top_p, min_p)
            assert abs(float(prob[n]) - p) <= 2.0 ** -23 * p, n

    for top_k in (1, 50, 1023, 1024, 1025):
        check(z, 1.1, top_k)
        check(z, 0.9, top_k, 0.9, 0.01)
    check(z, 1.0)
    check(z, 1.0, top_p=0.7)
    check(z, 1.3, min_p=0.05)
    check(z, 0.0)
    padded = torch.full((N, V + 9), math.nan, dtype=z.dtype, device="cuda")
    for first in (1, 3):
        padded[:, first:V + first] = z
        check(padded[:, first:V + first], 0.8, 30, 0.9)
        check(padded[:, first:V + first], 0.8)
