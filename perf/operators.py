"""Performance cases of the operators around the Hyena mixers: what a training step and a decoder call beside them.

* ``glr_fwd`` / ``glr_train`` / ``glr_step``: the gated linear recurrence ``s[t] = exp(g[t]) s[t-1] + k[t] v[t]``,
  ``y = q s``: forward (prefill), forward and gradients (training), one token of a batch of sequences (decoding);
* ``xent_eval`` / ``xent_train``: softmax cross entropy of ``x W^T`` over a vocabulary, the losses alone (scoring) or with
  the gradients of ``x`` and ``W``;
* ``adamw``: one AdamW step over the tensors of a model, states in 32 bits or in 8.

With ``own`` false, ``run`` computes them from elementary torch operations in 32 bits; with ``own`` true, it makes the
calls of the package.  Inputs are drawn on the GPU from the seed alone.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
IGNORED = -100          # a target that takes no part in the loss
BLOCK = 256             # elements that share a scale where the optimiser's states are held in 8 bits
TOP = 448.0             # largest value of the 8-bit floating type (e4m3)
TINY = 2.0 ** -100      # blocks whose largest magnitude is below this are held as zeros
BETA1, BETA2, EPS, LR, DECAY, STEP = 0.9, 0.95, 1e-8, 3e-4, 0.1, 100


def listed():
    return [
        # decoding: the next token of 64 sequences at the width of the 7B models; a call whose latency is what counts
        dict(name="glr_step_decode", op="glr_step", B=64, L=1, D=4096, group=1, dtype="bf16", carry=True, packed=False),
        # prefill of an 8K context at the width of the 7B models
        dict(name="glr_fwd_8k", op="glr_fwd", B=1, L=8192, D=4096, group=1, dtype="bf16", carry=False, packed=False),
        # a stretch of a longer stream: ragged batch and width, a decay for 8 channels, in and out states, fp32
        dict(name="glr_fwd_ragged_f32", op="glr_fwd", B=3, L=5003, D=1000, group=8, dtype="f32", carry=True, packed=False),
        # training at 8K context, one decay per channel
        dict(name="glr_train_8k", op="glr_train", B=1, L=8192, D=4096, group=1, dtype="bf16", carry=False, packed=False),
        # training on a packed 128K stream whose documents reset the memory, a decay per head of 16 channels
        dict(name="glr_train_128k_packed", op="glr_train", B=1, L=131072, D=1024, group=16, dtype="bf16", carry=True, packed=True),
        # scoring a few tokens against a large vocabulary: the weights' bytes are what counts
        dict(name="xent_eval_few_rows", op="xent_eval", N=8, V=65536, D=4096, dtype="bf16"),
        # training of a byte-level model: a small vocabulary and an 8K context
        dict(name="xent_train_bytes", op="xent_train", N=8192, V=512, D=4096, dtype="bf16"),
        # training with a large vocabulary
        dict(name="xent_train_64k", op="xent_train", N=8192, V=65536, D=4096, dtype="bf16"),
        # fp32 training of a small model with ragged sizes throughout
        dict(name="xent_train_ragged_f32", op="xent_train", N=1003, V=5003, D=1000, dtype="f32"),
        # the smallest model: few tensors, a call whose latency is what counts
        dict(name="adamw_small_f32", op="adamw", layers=1, D=256, bits=32, param="f32"),
        # a model of narrow layers, many of its tensors small (filters, biases), in bf16 with fp32 states and masters
        dict(name="adamw_narrow_bf16", op="adamw", layers=8, D=1024, bits=32, param="bf16+master"),
        # layers of the 7B models' width, in bf16 with fp32 masters and states in 8 bits
        dict(name="adamw_wide_8bit", op="adamw", layers=3, D=4096, bits=8, param="bf16+master"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["glr_step", "glr_fwd", "glr_fwd", "glr_train", "glr_train", "xent_eval", "xent_train", "xent_train",
                     "adamw", "adamw"])
    if op.startswith("glr"):
        group = rng.choice([1, 1, 1, 2, 3, 4, 8, 16, 16, 64, 128])
        D = group * max(1, round(_log(rng, 64, 4096) / group))
        B = rng.randint(1, 128) if op == "glr_step" else rng.randint(1, 8)
        L = 1 if op == "glr_step" else max(1, min(_log(rng, 1, 131072), 2 ** 27 // (B * D)))
        return dict(op=op, B=B, L=L, D=D, group=group, dtype=rng.choice(["bf16", "bf16", "f32"]),
                    carry=op == "glr_step" or rng.random() < 0.5, packed=op != "glr_step" and rng.random() < 0.3)
    if op.startswith("xent"):
        D = _log(rng, 128, 4096)
        D = D if rng.random() < 0.25 else -(-D // 8) * 8
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        N, V = _log(rng, 1, 8192), _log(rng, 256, 65536)
        if dtype == "f32":
            N = max(1, min(N, 2 ** 37 // (V * D)))
        return dict(op=op, N=N, V=V, D=D, dtype=dtype)
    D = _log(rng, 64, 4096)
    D = D if rng.random() < 0.25 else -(-D // 16) * 16
    return dict(op=op, layers=max(1, min(rng.randint(1, 12), 3 * 4096 * 4096 // (D * D))), D=D, bits=rng.choice([32, 8]),
                param=rng.choice(["f32", "bf16", "bf16+master"]))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    if case["op"].startswith("glr"):
        B, L, D, dtype = case["B"], case["L"], case["D"], DTYPES[case["dtype"]]
        shape = (B, D) if case["op"] == "glr_step" else (B, L, D)
        s = dict(case)
        s["q"], s["k"], s["v"] = (normal(*shape, dtype=dtype) for _ in range(3))
        # log decays with time constants from one step to a thousand
        g = -torch.exp(uniform(*shape[:-1], D // case["group"]) * math.log(1e-3))
        if case["packed"]:  # documents of 2000 tokens on average; their first steps forget everything
            g = torch.where(uniform(B, L, 1) < 1 / 2000, -math.inf, g)
        s["g"] = g.to(dtype)
        s["state"] = normal(B, D) if case["carry"] else None
        if case["op"] == "glr_train":
            s["dy"] = normal(*shape, dtype=dtype)
            s["dstate"] = normal(B, D) if case["carry"] else None
        return s
    if case["op"].startswith("xent"):
        N, V, D, dtype = case["N"], case["V"], case["D"], DTYPES[case["dtype"]]
        s = dict(case)
        s["x"], s["w"] = normal(N, D, dtype=dtype), normal(V, D, scale=2 / math.sqrt(D), dtype=dtype)
        target = torch.randint(0, V, (N,), generator=gen, device="cuda")
        s["target"] = torch.where(uniform(N) < 0.05, IGNORED, target)  # padding and prompts
        s["dloss"] = torch.full((N,), 1.0 / N, device="cuda")  # a mean over the rows
        return s
    return _prepare_adamw(case, normal, uniform)


def _shapes(case):
    """A layer: four projections, three featurizer filters, a medium filter per 16 channels, a bias."""
    D = case["D"]
    return case["layers"] * ([(D, D)] * 4 + [(D, 7)] * 3 + [(-(-D // 16), 128), (D,)])


def _prepare_adamw(case, normal, uniform):
    """Parameters, gradients and states lie in flat buffers, as a sharding trainer keeps them; a tensor begins at a multiple of
    256 elements, and what lies between two tensors is zero."""
    shapes = _shapes(case)
    sizes = [math.prod(x) for x in shapes]
    starts, total = [], 0
    for n in sizes:
        starts.append(total)
        total += -(-n // BLOCK) * BLOCK
    ends = [a + n for a, n in zip(starts, sizes)]
    # 1 inside a tensor and 0 between two: the running sum of +1 at each start and -1 at each end
    edge = torch.zeros(total + 1, device="cuda")
    edge.index_add_(0, torch.tensor(starts, device="cuda"), torch.ones(len(sizes), device="cuda"))
    edge.index_add_(0, torch.tensor(ends, device="cuda"), -torch.ones(len(sizes), device="cuda"))
    inside = edge.cumsum(0)[:total]
    s = dict(case)
    master = normal(total, scale=0.02) * inside
    dtype = torch.float32 if case["param"] == "f32" else torch.bfloat16
    s["p"] = master.to(dtype)
    s["master"] = master if case["param"] == "bf16+master" else None
    s["g"] = (normal(total, scale=1e-3) * inside).to(dtype)
    m, v = normal(total, scale=3e-4) * inside, (normal(total, scale=1e-3) * inside).square()
    if case["bits"] == 8:
        s["m"], s["m_scale"] = _to_8bit(m, False)
        s["v"], s["v_scale"] = _to_8bit(v.sqrt(), True)
    else:
        s["m"], s["v"], s["m_scale"], s["v_scale"] = m, v, None, None
    s["clip"] = torch.full((1,), 0.75, device="cuda")  # what clipping by the global norm multiplies the gradients with
    decay = [DECAY if len(x) == 2 and x[1] == case["D"] else 0.0 for x in shapes]  # projections decay, filters and biases do not
    per_block = torch.repeat_interleave(torch.tensor(decay), torch.tensor([-(-n // BLOCK) for n in sizes]))
    s["decay"] = per_block.cuda()[:, None]
    if own:
        import paper_2503_01868_amd as hy

        def tensors(flat, per=1):
            return None if flat is None else [flat[a // per:a // per + -(-n // per)] for a, n in zip(starts, sizes)]

        s["plan"] = hy.plan_adamw(tensors(s["p"]), tensors(s["g"]), tensors(s["m"]), tensors(s["v"]),
                                  masters=tensors(s["master"]), avg_scales=tensors(s["m_scale"], BLOCK),
                                  sq_scales=tensors(s["v_scale"], BLOCK), weight_decay=decay)
    return s


def run(s):
    if s["op"] == "glr_step":
        return _step_own(s) if own else _step(s)
    if s["op"].startswith("glr"):
        return _glr_own(s) if own else _glr(s)
    if s["op"].startswith("xent"):
        return _xent_own(s) if own else _xent(s)
    return _adamw_own(s) if own else _adamw(s)


# ---- the package's calls


def _step_own(s):
    import paper_2503_01868_amd as hy

    y = hy.hyena_glr_step(s["q"], s["k"], s["v"], s["g"], s["state"], s["group"])
    return {"y": y, "state": s["state"]}


def _glr_own(s):
    import paper_2503_01868_amd as hy

    if s["op"] == "glr_fwd":
        if not s["carry"]:
            return {"y": hy.hyena_glr_fwd(s["q"], s["k"], s["v"], s["g"], s["group"])}
        y, state, _ = hy.hyena_glr_fwd_carry(s["q"], s["k"], s["v"], s["g"], s["group"], state_in=s["state"])
        return {"y": y, "state": state}
    y, state, marks = hy.hyena_glr_fwd_carry(s["q"], s["k"], s["v"], s["g"], s["group"], state_in=s["state"],
                                             want_state=s["carry"], want_marks=True)
    dq, dk, dv, dg, dstate = hy.hyena_glr_bwd(s["dy"], s["q"], s["k"], s["v"], s["g"], s["group"], marks=marks,
                                              dstate_out=s["dstate"], want_dstate=s["carry"])
    return {"y": y, "state": state, "dq": dq, "dk": dk, "dv": dv, "dg": dg, "dstate": dstate}


def _xent_own(s):
    import paper_2503_01868_amd as hy

    loss, lse = hy.hyena_xent_fwd(s["x"], s["w"], s["target"])
    if s["op"] == "xent_eval":
        return {"loss": loss, "lse": lse}
    dx, dw = hy.hyena_xent_bwd(s["dloss"], s["x"], s["w"], s["target"], lse)
    return {"loss": loss, "lse": lse, "dx": dx, "dw": dw}


def _adamw_own(s):
    s["plan"](lr=LR, step=STEP, beta1=BETA1, beta2=BETA2, eps=EPS, grad_scale=s["clip"])
    return _adamw_outputs(s)


def _adamw_outputs(s):
    """The updated state.  The 8-bit type is a floating one: its values, and the scales that multiply them."""
    return {name: s[name] for name in ("p", "master", "m", "v", "m_scale", "v_scale") if s[name] is not None}


# ---- the plain forms


def _per_channel(g, group):
    return g if group == 1 else g.repeat_interleave(group, dim=-1)


def _step(s):
    a = torch.exp(_per_channel(s["g"].float(), s["group"]))
    s["state"].copy_(a * s["state"] + s["k"].float() * s["v"].float())
    return {"y": (s["q"].float() * s["state"]).to(s["q"].dtype), "state": s["state"]}


def _scan(a, x):
    """h[t] = a[t] h[t-1] + x[t] over dim 1 by doubling the reach of every step: log2(L) sweeps over all steps at once."""
    reach = 1
    while reach < x.shape[1]:
        x = torch.cat([x[:, :reach], x[:, reach:] + a[:, reach:] * x[:, :-reach]], 1)
        a = torch.cat([a[:, :reach], a[:, reach:] * a[:, :-reach]], 1)
        reach *= 2
    return x


def _glr(s):
    dtype, group = s["q"].dtype, s["group"]
    q, k, v, a = s["q"].float(), s["k"].float(), s["v"].float(), torch.exp(_per_channel(s["g"].float(), group))
    before = torch.zeros_like(q[:, 0]) if s["state"] is None else s["state"]
    x = k * v
    x[:, 0] += a[:, 0] * before
    h = _scan(a, x)
    out = {"y": (q * h).to(dtype)}
    if s["carry"]:
        out["state"] = h[:, -1].contiguous()
    if s["op"] == "glr_fwd":
        return out
    dy = s["dy"].float()
    x = q * dy
    if s["dstate"] is not None:
        x[:, -1] += s["dstate"]
    ahead = torch.cat([torch.zeros_like(a[:, :1]), a[:, 1:].flip(1)], 1)  # step t takes a[t + 1] m[t + 1]
    m = _scan(ahead, x.flip(1)).flip(1)
    kept = a * torch.cat([before[:, None], h[:, :-1]], 1)
    dg = (m * kept).reshape(*s["g"].shape, group).sum(-1)
    out.update(dq=(dy * h).to(dtype), dk=(m * v).to(dtype), dv=(m * k).to(dtype), dg=dg.to(dtype))
    if s["carry"]:
        out["dstate"] = a[:, 0] * m[:, 0]
    return out


def _xent(s):
    x, w, target = s["x"].float(), s["w"].float(), s["target"]
    z = x @ w.t()
    top = z.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(z - top).sum(1, keepdim=True))
    counts = (target >= 0) & (target < w.shape[0])
    at = torch.where(counts, target, 0)[:, None]
    loss = torch.where(counts, (lse - z.gather(1, at))[:, 0], 0.0)
    out = {"loss": loss, "lse": lse[:, 0]}
    if s["op"] == "xent_eval":
        return out
    p = torch.exp(z - lse)
    p.scatter_add_(1, at, torch.full_like(lse, -1.0))
    p *= torch.where(counts, s["dloss"], 0.0)[:, None]
    out.update(dx=(p @ w).to(s["x"].dtype), dw=(p.t() @ x).to(s["w"].dtype))
    return out


def _to_8bit(x, positive):
    """Blocks of 256 values as e4m3 numbers and a scale each: the largest magnitude becomes 448.  Of the roots of the second
    moments, which are divided by, none that is not zero becomes zero."""
    x = x.reshape(-1, BLOCK)
    top = x.abs().amax(1, keepdim=True)
    some = top >= TINY
    y = x * torch.where(some, torch.full_like(top, TOP) / top, 0.0)
    if positive:
        y = torch.where((x > 0) & some, y.clamp(min=2.0 ** -9), y)
    scale = torch.where(some, top * (1 / TOP), 0.0)
    return y.to(torch.float8_e4m3fn).reshape(-1), scale.reshape(-1)


def _adamw(s):
    p = (s["p"] if s["master"] is None else s["master"]).float().reshape(-1, BLOCK)
    g = s["g"].float().reshape(-1, BLOCK) * s["clip"]
    if s["bits"] == 8:
        m = s["m"].float().reshape(-1, BLOCK) * s["m_scale"][:, None]
        v = (s["v"].float().reshape(-1, BLOCK) * s["v_scale"][:, None]).square()
    else:
        m, v = s["m"].reshape(-1, BLOCK), s["v"].reshape(-1, BLOCK)
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    root = torch.sqrt(v)
    p = p * (1 - LR * s["decay"]) - (m * (LR / (1 - BETA1 ** STEP))) / (root * (1 / math.sqrt(1 - BETA2 ** STEP)) + EPS)
    p = p.reshape(-1)
    s["p"].copy_(p)
    if s["master"] is not None:
        s["master"].copy_(p)
    if s["bits"] == 8:
        s["m"], s["m_scale"] = _to_8bit(m, False)
        s["v"], s["v_scale"] = _to_8bit(root, True)
    else:
        s["m"], s["v"] = m.reshape(-1), v.reshape(-1)
    return _adamw_outputs(s)


# ---- what a pass cannot do without


def work(case):
    op = case["op"]
    if op.startswith("glr"):
        e = 4 if case["dtype"] == "f32" else 2
        n, ng = case["B"] * case["L"] * case["D"], case["B"] * case["L"] * case["D"] // case["group"]
        states = case["B"] * case["D"] * 4 * (2 if case["carry"] else 0)
        if op == "glr_train":  # q, k, v, dy in, y, dq, dk, dv out; g in, dg out
            return {"bytes": e * (8 * n + 2 * ng) + 2 * states, "flops": 14 * n}
        return {"bytes": e * (4 * n + ng) + states, "flops": 5 * n}
    if op.startswith("xent"):
        e = 4 if case["dtype"] == "f32" else 2
        N, V, D = case["N"], case["V"], case["D"]
        if op == "xent_train":  # x, w in, dx, dw out; the logits, dx, dw
            return {"bytes": 2 * e * (N + V) * D + 20 * N, "flops": 6.0 * N * V * D}
        return {"bytes": e * (N + V) * D + 16 * N, "flops": 2.0 * N * V * D}
    n = sum(math.prod(x) for x in _shapes(case))
    param = {"f32": 4 + 8, "bf16": 2 + 4, "bf16+master": 2 + 2 + 8}[case["param"]]  # gradient in, parameter (and master) in and out
    state = 4 + 4 * 4 / BLOCK if case["bits"] == 8 else 16
    return {"bytes": n * (param + state), "flops": 16 * n}


# ---- the definitions in 64 bits, step by step


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("glr"):
        return _exact_glr(case, s)
    if case["op"].startswith("xent"):
        return _exact_xent(case, s)
    return _exact_adamw(case, s)


def _exact_glr(case, s):
    one = case["op"] == "glr_step"
    q, k, v, g = (s[n].double()[:, None] if one else s[n].double() for n in "qkvg")
    B, L, D = q.shape
    decay = torch.exp(g)[..., None].expand(B, L, D // case["group"], case["group"]).reshape(B, L, D)
    h = s["state"].double() if s["state"] is not None else torch.zeros(B, D, dtype=torch.float64, device="cuda")
    kv, memory = k * v, torch.empty_like(q)
    before = torch.empty_like(q)
    for t in range(L):
        before[:, t] = h
        h = torch.addcmul(kv[:, t], decay[:, t], h)
        memory[:, t] = h
    y = q * memory
    if one:
        return {"y": y[:, 0], "state": h}
    out = {"y": y}
    if case["carry"]:
        out["state"] = h
    if case["op"] == "glr_fwd":
        return out
    dy = s["dy"].double()
    back = torch.empty_like(q)
    carry = s["dstate"].double() if s["dstate"] is not None else torch.zeros_like(h)
    qdy = q * dy
    for t in range(L - 1, -1, -1):
        back[:, t] = qdy[:, t] + carry
        carry = decay[:, t] * back[:, t]
    dg = (back * decay * before).reshape(B, L, D // case["group"], case["group"]).sum(3)
    out.update(dq=dy * memory, dk=back * v, dv=back * k, dg=dg)
    if case["carry"]:
        out["dstate"] = carry
    return out


def _exact_xent(case, s):
    N, V, D = case["N"], case["V"], case["D"]
    w = s["w"].double()
    grads = case["op"] == "xent_train"
    out = {n: torch.zeros(N, dtype=torch.float64, device="cuda") for n in ("loss", "lse")}
    if grads:
        out["dx"] = torch.zeros(N, D, dtype=torch.float64, device="cuda")
        out["dw"] = torch.zeros(V, D, dtype=torch.float64, device="cuda")
    for i in range(0, N, 1024):
        x, t = s["x"][i:i + 1024].double(), s["target"][i:i + 1024]
        z = torch.mm(x, w.t().contiguous())
        lse = torch.logsumexp(z, 1)
        out["lse"][i:i + 1024] = lse
        rows = torch.nonzero((t >= 0) & (t < V))[:, 0]
        out["loss"][i + rows] = lse[rows] - z[rows, t[rows]]
        if grads:
            p = torch.softmax(z[rows], 1)
            p[torch.arange(len(rows), device="cuda"), t[rows]] -= 1.0
            p = p * s["dloss"][i + rows].double()[:, None]
            out["dx"][i + rows] = torch.mm(p, w)
            out["dw"] += torch.mm(p.t().contiguous(), x[rows])
    return out


def _exact_adamw(case, s):
    n = s["p"].numel() // BLOCK
    out = {name: [] for name in ("p", "master", "m", "v", "m_scale", "v_scale") if s[name] is not None}
    for i in range(0, n, 1 << 17):  # by pieces of 32 Mi elements
        at = slice(i * BLOCK, min(n, i + (1 << 17)) * BLOCK)
        p = (s["p"] if s["master"] is None else s["master"])[at].double()
        g = s["g"][at].double() * float(s["clip"])
        m, v = s["m"][at].double(), s["v"][at].double()
        if case["bits"] == 8:
            m = m * s["m_scale"][i:i + (1 << 17)].double().repeat_interleave(BLOCK)
            v = (v * s["v_scale"][i:i + (1 << 17)].double().repeat_interleave(BLOCK)) ** 2
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g ** 2
        decay = s["decay"][i:i + (1 << 17)].double().expand(-1, BLOCK).reshape(-1)
        m_hat, v_hat = m / (1 - BETA1 ** STEP), v / (1 - BETA2 ** STEP)
        p = p - LR * (decay * p + m_hat / (v_hat.sqrt() + EPS))
        out["p"].append(p)
        if s["master"] is not None:
            out["master"].append(p)
        if case["bits"] == 8:
            for name, x in (("m", m), ("v", v.sqrt())):
                top = x.abs().view(-1, BLOCK).max(1).values
                unit = torch.where(top >= TINY, top / TOP, 0.0)
                y = torch.where(unit[:, None] > 0, x.view(-1, BLOCK) / unit[:, None], 0.0).reshape(-1)
                # e4m3: four significant bits, steps of 2^-9 below 2^-6
                step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
                held = torch.round(y / step) * step
                if name == "v":
                    held = torch.where((y > 0) & (held == 0), 2.0 ** -9, held)
                out[name].append(held)
                out[name + "_scale"].append(unit)
        else:
            out["m"].append(m)
            out["v"].append(v)
    return {name: torch.cat(parts) for name, parts in out.items()}
