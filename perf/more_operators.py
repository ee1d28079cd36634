"""Performance cases of what a recurrent block and a decoder need beside the mixers of ``operators.py``.

* ``la_fwd`` / ``la_train`` / ``la_step``: linear attention with a decay for each head, ``S[t] = exp(g[t]) S[t-1] + k[t]^T v[t]``,
  ``y[t] = scale q[t] S[t]``: forward (prefill), forward and gradients (training), one token of a batch of sequences (decoding);
* ``norm`` / ``norm8`` / ``norm_train``: root-mean-square norm with the residual's addition, in the activations' type, with an
  8-bit output and a scale per row, forward and gradients;
* ``sample``: the next token of every row of logits by temperature, top-k, top-p and min-p, from given random numbers.

With ``own`` false, ``run`` computes them from elementary torch operations; with ``own`` true, it makes the calls of the package.
Inputs are drawn on the GPU from the seed alone.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CHUNK = 64       # steps that the plain form of the linear attention takes together
FORGETS = -87.0  # a log decay below it forgets everything before its step
EPS = 1e-6
TOP = 448.0      # largest value of the 8-bit floating type (e4m3)
TINY = 2.0 ** -100  # rows whose largest magnitude is below this are held as zeros


def listed():
    return [
        # decoding: the next token of 64 sequences at the width of the 7B models, 32 heads; the states are what counts
        dict(name="la_step_decode", op="la_step", B=64, L=1, H=32, group=1, dk=128, dv=128, dtype="bf16", carry=True, packed=False),
        # prefill of an 8K context at that width
        dict(name="la_fwd_8k", op="la_fwd", B=1, L=8192, H=32, group=1, dk=128, dv=128, dtype="bf16", carry=False, packed=False),
        # a stretch of a longer stream: ragged length and heads, q and k shared by three heads, in and out states, fp32
        dict(name="la_fwd_ragged_f32", op="la_fwd", B=3, L=1003, H=6, group=3, dk=40, dv=72, dtype="f32", carry=True, packed=False),
        # training at 8K context
        dict(name="la_train_8k", op="la_train", B=1, L=8192, H=32, group=1, dk=128, dv=128, dtype="bf16", carry=False, packed=False),
        # training on a packed 32K stream whose documents reset the memory, q and k shared by four heads
        dict(name="la_train_32k_packed", op="la_train", B=1, L=32768, H=16, group=4, dk=64, dv=128, dtype="bf16", carry=True, packed=True),
        # decoding: the norm in front of a mixer for 64 sequences; a call whose latency is what counts
        dict(name="norm_decode", op="norm", N=64, D=4096, dtype="bf16", residual=True, weight=True),
        # prefill of an 8K context, for a projection that takes 8-bit rows
        dict(name="norm8_8k", op="norm8", N=8192, D=4096, dtype="bf16", residual=True, weight=True),
        # training at 8K context
        dict(name="norm_train_8k", op="norm_train", N=8192, D=4096, dtype="bf16", residual=True, weight=True),
        # fp32 training of a small model, ragged rows
        dict(name="norm_train_ragged_f32", op="norm_train", N=1003, D=1000, dtype="f32", residual=True, weight=True),
        # a byte-level model writes: one row, the smallest vocabulary
        dict(name="sample_bytes", op="sample", N=1, V=512, dtype="f32", limits="all"),
        # decoding of 64 sequences over a large vocabulary
        dict(name="sample_decode", op="sample", N=64, V=65536, dtype="bf16", limits="all"),
        # many sequences at once over the largest vocabulary, fp32 logits
        dict(name="sample_many", op="sample", N=512, V=131072, dtype="f32", limits="all"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["la_step", "la_fwd", "la_fwd", "la_train", "la_train", "norm", "norm8", "norm_train", "norm_train", "sample", "sample"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op.startswith("la"):
        dk = rng.choice([16, 32, 64, 64, 128, 128, rng.randint(8, 128)])
        dv = rng.choice([16, 32, 64, 64, 128, 128, 256, rng.randint(8, 256)])
        group = rng.choice([1, 1, 1, 2, 3, 4])
        H = group * rng.randint(1, max(1, 32 // group))
        B = rng.randint(1, 64) if op == "la_step" else rng.randint(1, 8)
        if op == "la_step":
            return dict(op=op, B=max(1, min(B, 2 ** 25 // (H * dk * dv))), L=1, H=H, group=group, dk=dk, dv=dv, dtype=dtype, carry=True, packed=False)
        # no more states and elements than the 8K cases have
        most = min(2 ** 24 // (B * H * max(dk, dv)), 2 ** 31 // (B * H * dk * dv), 32768)
        return dict(op=op, B=B, L=max(1, min(_log(rng, 1, 32768), most)), H=H, group=group, dk=dk, dv=dv, dtype=dtype,
                    carry=rng.random() < 0.5, packed=rng.random() < 0.3)
    if op.startswith("norm"):
        D = _log(rng, 64, 8192)
        D = D if rng.random() < 0.25 else -(-D // 16) * 16
        return dict(op=op, N=max(1, min(_log(rng, 1, 16384), 2 ** 24 // D)), D=D, dtype=dtype, residual=rng.random() < 0.7,
                    weight=rng.random() < 0.8)
    V = _log(rng, 256, 131072)
    V = V if rng.random() < 0.5 else -(-V // 64) * 64
    return dict(op=op, N=max(1, min(_log(rng, 1, 512), 2 ** 25 // V)), V=V, dtype=dtype,
                limits=rng.choice(["all", "all", "top_k", "top_p", "min_p", "none", "greedy"]))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)

    def uniform(*shape, lo=0.0, hi=1.0):
        return torch.rand(*shape, generator=gen, device="cuda") * (hi - lo) + lo

    s, dtype = dict(case), DTYPES[case["dtype"]]
    if case["op"].startswith("la"):
        B, H, dk, dv = case["B"], case["H"], case["dk"], case["dv"]
        at = (B,) if case["op"] == "la_step" else (B, case["L"])
        s["q"], s["k"] = (normal(*at, H // case["group"], dk, dtype=dtype) for _ in range(2))
        s["v"] = normal(*at, H, dv, dtype=dtype)
        # log decays with time constants from one step to a thousand
        g = -torch.exp(uniform(*at, H) * math.log(1e-3))
        if case["packed"]:  # documents of 2000 tokens on average; their first steps forget everything
            g = torch.where(uniform(*at, 1) < 1 / 2000, -math.inf, g)
        s["g"], s["scale"] = g.to(dtype), 1 / math.sqrt(dk)
        s["state"] = normal(B, H, dk, dv) if case["carry"] else None
        if case["op"] == "la_train":
            s["dy"] = normal(*at, H, dv, dtype=dtype)
            s["dstate"] = normal(B, H, dk, dv) if case["carry"] else None
        return s
    if case["op"].startswith("norm"):
        N, D = case["N"], case["D"]
        s["x"] = normal(N, D, dtype=dtype)
        s["residual"] = normal(N, D, scale=2.0, dtype=dtype) if case["residual"] else None
        s["w"] = (1 + normal(D, scale=0.1)).to(dtype) if case["weight"] else None
        if case["op"] == "norm_train":
            s["dy"] = normal(N, D, dtype=dtype)
            s["dtotal"] = normal(N, D, dtype=dtype) if case["residual"] else None  # what comes back along the residual
        return s
    N, limits = case["N"], case["limits"]
    # logits of a trained model: most words far below the likeliest
    s["logits"] = normal(N, case["V"], scale=2.5, dtype=dtype)
    s["u"] = uniform(N)
    # every sequence has the settings of its own user
    s["temperature"] = torch.zeros(N, device="cuda") if limits == "greedy" else uniform(N, lo=0.5, hi=1.5)
    top_k = torch.randint(1, min(case["V"], 1000) + 1, (N,), generator=gen, device="cuda", dtype=torch.int32)
    s["top_k"] = top_k if limits in ("all", "top_k") else None
    s["top_p"] = uniform(N, lo=0.5, hi=1.0) if limits in ("all", "top_p") else None
    s["min_p"] = uniform(N, lo=0.001, hi=0.1) if limits in ("all", "min_p") else None
    return s


def run(s):
    if s["op"] == "la_step":
        return _step_own(s) if own else _step(s)
    if s["op"].startswith("la"):
        return _la_own(s) if own else _la(s)
    if s["op"].startswith("norm"):
        return _norm_own(s) if own else _norm(s)
    return _sample_own(s) if own else _sample(s)


# ---- the package's calls


def _step_own(s):
    import paper_2503_01868_amd as hy

    y = hy.hyena_la_step(s["q"], s["k"], s["v"], s["g"], s["state"], scale=s["scale"])
    return {"y": y, "state": s["state"]}


def _la_own(s):
    import paper_2503_01868_amd as hy

    if s["op"] == "la_fwd":
        if not s["carry"]:
            return {"y": hy.hyena_la_fwd(s["q"], s["k"], s["v"], s["g"], scale=s["scale"])}
        y, state, _ = hy.hyena_la_fwd_carry(s["q"], s["k"], s["v"], s["g"], scale=s["scale"], state_in=s["state"])
        return {"y": y, "state": state}
    y, state, marks = hy.hyena_la_fwd_carry(s["q"], s["k"], s["v"], s["g"], scale=s["scale"], state_in=s["state"],
                                            want_state=s["carry"], want_marks=True)
    dq, dk, dv, dg, dstate = hy.hyena_la_bwd(s["dy"], s["q"], s["k"], s["v"], s["g"], scale=s["scale"], marks=marks,
                                             dstate_out=s["dstate"], want_dstate=s["carry"])
    return {"y": y, "state": state, "dq": dq, "dk": dk, "dv": dv, "dg": dg, "dstate": dstate}


def _norm_own(s):
    import paper_2503_01868_amd as hy

    if s["op"] == "norm8":
        y, scale, total, _ = hy.hyena_rmsnorm_fwd_8bit(s["x"], s["w"], residual=s["residual"], eps=EPS)
        return {"y": y, "scale": scale, "total": total if s["residual"] is not None else None}
    y, total, rstd = hy.hyena_rmsnorm_fwd(s["x"], s["w"], residual=s["residual"], eps=EPS, want_rstd=s["op"] == "norm_train")
    out = {"y": y, "total": total if s["residual"] is not None else None}
    if s["op"] == "norm":
        return out
    dx, dw = hy.hyena_rmsnorm_bwd(s["dy"], total, rstd, s["w"], dtotal=s["dtotal"])
    out.update(rstd=rstd, dx=dx, dw=dw)
    return out


def _sample_own(s):
    import paper_2503_01868_amd as hy

    token, prob = hy.hyena_sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    return {"token": token, "prob": prob}


# ---- the plain forms


def _per_head(x, group):
    return x if group == 1 else x.repeat_interleave(group, dim=-2)


def _step(s):
    q, k = (_per_head(s[n].float(), s["group"]) for n in "qk")
    a = torch.exp(s["g"].float())[..., None, None]
    s["state"].copy_(a * s["state"] + k[..., :, None] * s["v"].float()[..., None, :])
    y = s["scale"] * (q[..., :, None] * s["state"]).sum(-2)
    return {"y": y.to(s["v"].dtype), "state": s["state"]}


def _chunks(x, n):
    """[B, L, H, d] as [B, H, chunks, CHUNK, d], zeros behind the last step."""
    B, L, H, d = x.shape
    x = torch.cat([x, x.new_zeros(B, n * CHUNK - L, H, d)], 1)
    return x.reshape(B, n, CHUNK, H, d).permute(0, 3, 1, 2, 4).contiguous()


def _rows(x, L):
    """_chunks the other way."""
    B, H, n, c, d = x.shape
    return x.permute(0, 2, 3, 1, 4).reshape(B, n * c, H, d)[:, :L]


def _between(log_hi, log_lo, doc_hi, doc_lo):
    """Products of decays as exp of differences of running sums of their logarithms, in 64 bits; zero across a reset.  (Of pairs
    in the wrong order, which count for nothing, no infinities.)"""
    return torch.where(doc_hi == doc_lo, torch.exp((log_hi - log_lo).clamp(max=0.0)), 0.0).float()


def _la(s):
    """Products inside chunks, and the chunks' states from one matrix of decays between chunks."""
    dtype, group, scale = s["q"].dtype, s["group"], s["scale"]
    B, L, H, dv = s["v"].shape
    dk, n = s["q"].shape[-1], -(-L // CHUNK)
    q, k = (_chunks(_per_head(s[name].float(), group), n) for name in "qk")
    v = _chunks(s["v"].float(), n)
    g = s["g"].double()
    forgets = g < FORGETS
    b = _chunks(torch.where(forgets, 0.0, g).cumsum(1)[..., None], n)[..., 0]  # [B, H, n, C]
    doc = _chunks(forgets.cumsum(1)[..., None], n)[..., 0]
    behind = torch.arange(n * CHUNK, device="cuda").reshape(n, CHUNK) >= L  # (padding: as the last step, and nothing in it)
    last_b, last_doc = (x.flatten(2)[:, :, L - 1:L, None] for x in (b, doc))
    b, doc = torch.where(behind, last_b, b), torch.where(behind, last_doc, doc)
    first = torch.zeros_like(b[:, :, :1, :1])  # in front of the first step
    start_b = torch.cat([first, b[:, :, :-1, -1:]], 2)   # in front of every chunk: [B, H, n, 1]
    start_doc = torch.cat([first.long(), doc[:, :, :-1, -1:]], 2)
    end_b, end_doc = b[..., -1:], doc[..., -1:]
    before = torch.zeros(B, H, dk, dv, device="cuda") if s["state"] is None else s["state"]

    at = torch.arange(CHUNK, device="cuda")
    inside = _between(b[..., :, None], b[..., None, :], doc[..., :, None], doc[..., None, :]) * (at[:, None] >= at[None, :])
    from_start = _between(b, start_b, doc, start_doc)[..., None]     # chunk's start to a step
    to_end = _between(end_b, b, end_doc, doc)[..., None]             # a step to the chunk's end
    local = (k * to_end).transpose(-1, -2) @ v                      # what a chunk adds: [B, H, n, dk, dv]
    c = torch.arange(n, device="cuda")
    hop = _between(start_b, end_b.transpose(-1, -2), start_doc, end_doc.transpose(-1, -2)) * (c[:, None] > c[None, :])
    from_first = _between(start_b, first, start_doc, first.long())[..., None]
    start = (hop @ local.flatten(3)).unflatten(3, (dk, dv)) + from_first * before[:, :, None]
    p = (q @ k.transpose(-1, -2)) * (inside * scale)
    far = (q @ start) * (from_start * scale)
    out = {"y": _rows(p @ v + far, L).to(dtype)}
    if s["carry"]:
        whole = _between(end_b[:, :, -1], start_b[:, :, -1], end_doc[:, :, -1], start_doc[:, :, -1])[..., None]
        out["state"] = whole * start[:, :, -1] + local[:, :, -1]
    if s["op"] == "la_fwd":
        return out
    dy = _chunks(s["dy"].float(), n)
    behind_all = torch.zeros_like(before) if s["dstate"] is None else s["dstate"]
    # gradients of the states at the chunks' ends
    back = (q * (from_start * scale)).transpose(-1, -2) @ dy
    to_last = _between(end_b[:, :, -1:], end_b, end_doc[:, :, -1:], end_doc)[..., None]
    end = (hop.transpose(-1, -2) @ back.flatten(3)).unflatten(3, (dk, dv)) + to_last * behind_all[:, :, None]
    dp = (dy @ v.transpose(-1, -2)) * (inside * scale)
    dq_far = (dy @ start.transpose(-1, -2)) * (from_start * scale)
    dk_far = (v @ end.transpose(-1, -2)) * to_end
    dq, dk_ = dp @ k + dq_far, dp.transpose(-1, -2) @ q + dk_far
    dv_ = p.transpose(-1, -2) @ dy + (k @ end) * to_end
    # dg[t]: what pairs of steps on both sides of decay t say to each other, one or both of them perhaps in another chunk
    w = (p * (dy @ v.transpose(-1, -2))).double()
    near = w.sum(-1) - w.sum(-2)
    rows, columns = (q * dq_far).double().sum(-1), (k * dk_far).double().sum(-1)
    across = (_between(end_b, start_b, end_doc, start_doc)[..., None] * start * end).double().sum((-1, -2))[..., None]
    dg = (near + rows).flip(-1).cumsum(-1).flip(-1) + (columns.cumsum(-1) - columns) + across
    dg = torch.where(_chunks(forgets[..., None], n)[..., 0], 0.0, dg)

    def shared(x):
        x = _rows(x, L)
        return x.reshape(B, L, H // group, group, dk).sum(3).to(dtype)

    out.update(dq=shared(dq), dk=shared(dk_), dv=_rows(dv_, L).to(dtype), dg=_rows(dg[..., None], L)[..., 0].to(dtype))
    if s["carry"]:
        whole = _between(end_b[:, :, 0], start_b[:, :, 0], end_doc[:, :, 0], start_doc[:, :, 0])[..., None]
        out["dstate"] = whole * end[:, :, 0] + back[:, :, 0]
    return out


def _norm(s):
    dtype = s["x"].dtype
    x, w = s["x"].float(), 1.0 if s["w"] is None else s["w"].float()
    h = x if s["residual"] is None else (x + s["residual"].float()).to(dtype).float()
    rstd = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
    total = None if s["residual"] is None else h.to(dtype)
    if s["op"] == "norm8":
        u = h * w
        top = u.abs().amax(1, keepdim=True)
        some = top >= TINY
        up = torch.where(some, torch.full_like(top, TOP) / top, 0.0)
        scale = torch.where(some, top * (1 / TOP) * rstd, 0.0)
        return {"y": (u * up).to(torch.float8_e4m3fn), "scale": scale[:, 0], "total": total}
    out = {"y": (h * rstd * w).to(dtype), "total": total}
    if s["op"] == "norm":
        return out
    dy = s["dy"].float()
    wdy = dy * w
    dx = rstd * (wdy - h * (rstd * rstd * (wdy * h).mean(1, keepdim=True)))
    if s["dtotal"] is not None:
        dx = dx + s["dtotal"].float()
    out.update(rstd=rstd[:, 0], dx=dx.to(dtype), dw=None if s["w"] is None else (dy * h * rstd).sum(0).to(dtype))
    return out


def _sample(s):
    """Sorted by size, ties by index; 64 bits, for words next to a border."""
    z, N = s["logits"].double(), len(s["u"])
    T = s["temperature"].double()[:, None]
    z, order = torch.sort(z, dim=1, descending=True, stable=True)
    far = (z - z[:, :1]) / torch.where(T > 0, T, 1.0)
    weight = torch.exp(far)
    rank = torch.arange(z.shape[1], device="cuda")[None]
    kept = (T > 0) | (rank == 0)
    if s["top_k"] is not None:
        kept = kept & (rank < s["top_k"][:, None])
    if s["top_p"] is not None:
        some = torch.where(kept, weight, 0.0)
        above = some.cumsum(1) - some  # the weight of what is likelier
        kept = kept & ((above < s["top_p"].double()[:, None] * some.sum(1, keepdim=True)) | (rank == 0))
    if s["min_p"] is not None:
        kept = kept & (weight >= s["min_p"].double()[:, None])
    weight = torch.where(kept, weight, 0.0)
    weight = torch.zeros_like(weight).scatter_(1, order, weight)  # in the vocabulary's order again
    upto = weight.cumsum(1)
    total = upto[:, -1:]
    token = (upto <= s["u"].double()[:, None] * total).sum(1)
    last = torch.where(weight > 0, rank, 0).amax(1)
    token = torch.minimum(token, last)
    prob = (weight.gather(1, token[:, None]) / total)[:, 0].float()
    return {"token": token, "prob": prob}


# ---- what a pass cannot do without


def work(case):
    op, e = case["op"], 4 if case["dtype"] == "f32" else 2
    if op.startswith("la"):
        rows, dk, dv = case["B"] * case["L"], case["dk"], case["dv"]
        qk, v, g = rows * case["H"] // case["group"] * dk, rows * case["H"] * dv, rows * case["H"]
        states = case["B"] * case["H"] * dk * dv * 4 * (2 if case["carry"] else 0)
        if op == "la_train":  # q, k, v, g, dy in, y, dq, dk, dv, dg out; S, y, M, dq, dk, dv
            return {"bytes": e * (4 * qk + 4 * v + 2 * g) + 2 * states, "flops": 12 * g * dk * dv}
        return {"bytes": e * (2 * qk + 2 * v + g) + states, "flops": 4 * g * dk * dv}
    if op.startswith("norm"):
        n, extra = case["N"] * case["D"], 2 if case["residual"] else 0
        if op == "norm_train":  # x (or the sum), dy in, y, dx out; residual in, sum out; the sum and its gradient in again
            return {"bytes": e * n * (4 + extra + (1 if extra else 0)) + 4 * case["N"], "flops": 14 * n}
        if op == "norm8":
            return {"bytes": n * (e + 1 + e * extra) + 4 * case["N"], "flops": 6 * n}
        return {"bytes": e * n * (2 + extra), "flops": 5 * n}
    return {"bytes": e * case["N"] * case["V"] + 28 * case["N"], "flops": 4 * case["N"] * case["V"]}


# ---- the definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("la"):
        return _exact_la(case, s)
    return _exact_norm(case, s) if case["op"].startswith("norm") else _exact_sample(case, s)


def _exact_la(case, s):
    """Step by step.  The gradient of a log decay from <S, dS> before and behind a step, whose difference the step's own terms are."""
    one, group, scale = case["op"] == "la_step", case["group"], s["scale"]
    q, k, v, g = (s[n].double()[:, None] if one else s[n].double() for n in "qkvg")
    B, L, H, dv = v.shape
    q, k = (x[..., None, :].expand(*x.shape[:-1], group, x.shape[-1]).flatten(2, 3) for x in (q, k))
    a = torch.exp(g)[..., None, None]
    S = s["state"].double() if s["state"] is not None else torch.zeros(B, H, q.shape[-1], dv, dtype=torch.float64, device="cuda")
    train = case["op"] == "la_train"
    dy = s["dy"].double() if train else None
    y, dq = torch.empty_like(v), torch.empty_like(q)
    for t in range(L):
        S = a[:, t] * S
        S = S + k[:, t, :, :, None] * v[:, t, :, None, :]
        y[:, t] = scale * (q[:, t, :, :, None] * S).sum(2)
        if train:
            dq[:, t] = scale * (S * dy[:, t, :, None, :]).sum(3)
    if one:
        return {"y": y[:, 0], "state": S}
    out = {"y": y}
    if case["carry"]:
        out["state"] = S
    if not train:
        return out
    M = s["dstate"].double() if s["dstate"] is not None else torch.zeros_like(S)  # with respect to the state behind step t
    dk, dv_, dg = torch.empty_like(k), torch.empty_like(v), torch.empty_like(g)
    both = (S * M).sum((2, 3))
    for t in range(L - 1, -1, -1):
        M = M + scale * q[:, t, :, :, None] * dy[:, t, :, None, :]
        dk[:, t] = (M * v[:, t, :, None, :]).sum(3)
        dv_[:, t] = (M * k[:, t, :, :, None]).sum(2)
        both = both + (q[:, t] * dq[:, t]).sum(2) - (k[:, t] * dk[:, t]).sum(2)
        both = torch.where(a[:, t, :, 0, 0] > 0, both, 0.0)
        dg[:, t] = both
        M = a[:, t] * M
    out.update(dq=dq.unflatten(2, (H // group, group)).sum(3), dk=dk.unflatten(2, (H // group, group)).sum(3), dv=dv_, dg=dg)
    if case["carry"]:
        out["dstate"] = M
    return out


def _exact_norm(case, s):
    x, w = s["x"].double(), torch.ones(case["D"], dtype=torch.float64, device="cuda") if s["w"] is None else s["w"].double()
    if s["residual"] is not None:  # the sum is rounded: it is what the next layer adds to
        x = (x + s["residual"].double()).to(s["x"].dtype).double()
    total = x if s["residual"] is not None else None
    size = torch.sqrt(x.pow(2).sum(1, keepdim=True) / case["D"] + EPS)
    if case["op"] == "norm8":
        u = x * w
        unit = u.abs().amax(1, keepdim=True) / TOP
        y = torch.where(unit > 0, u / unit, 0.0)
        # e4m3: four significant bits, steps of 2^-9 below 2^-6
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
        return {"y": torch.round(y / step) * step, "scale": (unit / size)[:, 0], "total": total}
    out = {"y": x / size * w, "total": total}
    if case["op"] == "norm":
        return out
    dy, unit = s["dy"].double(), x / size
    inner = ((dy * w) * unit).sum(1, keepdim=True) / case["D"]
    dx = (dy * w - unit * inner) / size
    if s["dtotal"] is not None:
        dx = dx + s["dtotal"].double()
    out.update(rstd=1 / size[:, 0], dx=dx, dw=None if s["w"] is None else (dy * unit).sum(0))
    return out


def _exact_sample(case, s):
    """Row by row, by selecting instead of sorting everything."""
    tokens, probs = [], []
    for i in range(case["N"]):
        z, T = s["logits"][i].double(), float(s["temperature"][i])
        if T == 0:
            tokens.append(int(torch.nonzero(z == z.max())[0]))
            probs.append(1.0)
            continue
        w = torch.softmax(z / T, 0)
        order = torch.argsort(z, descending=True, stable=True)
        if s["top_k"] is not None:
            order = order[:int(s["top_k"][i])]
        if s["top_p"] is not None:
            upto = w[order].cumsum(0)
            order = order[:int((upto < float(s["top_p"][i]) * upto[-1]).sum()) + 1]
        if s["min_p"] is not None:
            order = order[w[order] >= float(s["min_p"][i]) * w.max()]
        words = order.sort().values
        upto = w[words].cumsum(0)
        at = min(int((upto <= float(s["u"][i]) * upto[-1]).sum()), len(words) - 1)
        tokens.append(int(words[at]))
        probs.append(float(w[words[at]] / upto[-1]))
    return {"token": torch.tensor(tokens, device="cuda"), "prob": torch.tensor(probs, dtype=torch.float64, device="cuda")}
