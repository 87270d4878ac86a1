"""The gated delta rule and the AdamW step: workloads, plain forms and 64-bit definitions.

The gated delta rule keeps a matrix state per value head, S (dk x dv), and per step
    S~ = exp(g_t) S_{t-1},  u_t = beta_t (v_t - S~^T k_t),  S_t = S~ + k_t u_t^T,  o_t = scale S_t^T q_t.
Kinds of case:
    "steps"    K recurrent steps on the states of B rows (serving)
    "prefill"  whole sequences, outputs and last states (serving a history)
    "train"    whole sequences, outputs and the gradients of every input (training)
Rows of their own lengths are left-padded: row b is its last lengths[b] steps, the padding's
outputs and gradients are zero.
    "adamw"    one AdamW step over a model's tensors, the moments in float32 or in 8 bits
               (float8 e4m3 with a float32 scale for every 256 values; the second moment as its root)
"""
import math

import torch

own = False

CHUNK = 64
BLOCK = 256
E4M3_MAX = 448.0
E4M3_TINY = 2.0 ** -9


def listed():
    return [
        # the latest behavior of a single user, answered at once
        gdr("steps_one_row", "steps", 1, 1, 1, 2, 64, 64, "bf16"),
        # one new behavior for each of many users
        gdr("steps_many_rows", "steps", 1024, 1, 2, 4, 128, 128, "bf16"),
        # a few behaviors at once, float32, an odd number of users
        gdr("steps_burst_f32", "steps", 333, 5, 2, 2, 64, 128, "f32"),
        # a handful of short histories
        gdr("prefill_short_f32", "prefill", 3, 37, 2, 2, 64, 64, "f32", state=True),
        # histories of their own lengths (an empty one and one of a single step among them)
        gdr("prefill_ragged", "prefill", 32, 1000, 2, 4, 128, 128, "bf16", ragged=True, state=True),
        # one very long history
        gdr("prefill_long", "prefill", 1, 32768, 4, 8, 128, 128, "bf16", state=True),
        # a training batch of short sequences of their own lengths
        gdr("train_batch", "train", 2048, 50, 2, 2, 64, 64, "bf16", ragged=True),
        # odd sizes, float32, carried states with their gradients, shared key heads
        gdr("train_odd_f32", "train", 4, 333, 1, 2, 64, 128, "f32", state=True),
        # long sequences, 8 x 32768 x 512
        gdr("train_long", "train", 8, 32768, 4, 4, 128, 128, "bf16"),
        # a small recommender: two layers of width 64 and its item table
        adamw("adamw_small_f32", 64, 2, 1001, "f32", 32, False),
        # a large one: bfloat16 weights with float32 masters
        adamw("adamw_large_master", 512, 24, 200003, "bf16", 32, True),
        # bfloat16 weights, 8-bit moments
        adamw("adamw_8bit", 512, 12, 100003, "bf16", 8, False),
    ]


def gdr(name, kind, B, L, hk, hv, dk, dv, io, ragged=False, state=False):
    return dict(name=name, kind=kind, B=B, L=L, hk=hk, hv=hv, dk=dk, dv=dv, io=io, ragged=ragged, state=state)


def adamw(name, width, layers, items, io, bits, master):
    return dict(name=name, kind="adamw", width=width, layers=layers, items=items, io=io, bits=bits, master=master)


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["steps", "prefill", "train", "train", "adamw"])
    io = rng.choice(["bf16", "bf16", "f32"])
    if kind == "adamw":
        master = io == "bf16" and rng.random() < 0.5
        c = adamw("", 8 * log(2, 64), log(1, 24), log(100, 200003), io, rng.choice([32, 8]), master)
    else:
        hk, group = rng.choice([1, 2, 4]), rng.choice([1, 1, 2])
        dk, dv = rng.choice([64, 128]), rng.choice([64, 128])
        row = hk * group * dk * dv
        if kind == "steps":
            K = log(1, 8)
            c = gdr("", kind, log(1, max(1, min(4096, 2 ** 26 // row))), K, hk, hk * group, dk, dv, io)
        else:
            L = log(1, 16384)
            most = 2 ** 27 if kind == "train" else 2 ** 25
            B = log(1, max(1, min(2048, most // (hk * group * 128 * (L + 63)))))
            c = gdr("", kind, B, L, hk, hk * group, dk, dv, io, rng.random() < 0.5, kind == "prefill" or rng.random() < 0.3)
    c.pop("name")
    return c


def _type(case):
    return torch.bfloat16 if case["io"] == "bf16" else torch.float32


def _shapes(case):
    """The tensors of a recommender of gated recurrent layers: projections, convolution, decay, norms, item table."""
    d, e = case["width"], 2 * case["width"]
    layer = [(2 * e, d), (2 * e,), (e, 1, 4), (e,), (2 * e, e), (2 * e,), (d, e), (d,), (e,), (d,), (d,)]
    return layer * case["layers"] + [(case["items"], d), (d,), (d,)]


def _places(case):
    """Where each tensor begins in a flat buffer (multiples of BLOCK), and the buffer's size."""
    at, begins = 0, []
    for s in _shapes(case):
        begins.append(at)
        at += -(-math.prod(s) // BLOCK) * BLOCK
    return begins, at


def _views(flat, case, begins, per=1):
    return [flat[b // per:b // per + -(-math.prod(s) // per)].view(*(s if per == 1 else (-1,))) for b, s in zip(begins, _shapes(case))]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    def uniform(*shape):
        return torch.rand(*shape, device="cuda", generator=gen)

    io = _type(case)
    if case["kind"] == "adamw":
        begins, n = _places(case)
        real = torch.zeros(n, device="cuda")
        for v in _views(real, case, begins):
            v.fill_(1.0)
        size = 0.05 * torch.exp(1.5 * normal(n // BLOCK)).repeat_interleave(BLOCK)  # a gradient scale for each block
        s = dict(case=case, step=100, p=(0.05 * normal(n) * real).to(io), g=(size * normal(n) * real).to(io))
        m, r = 0.3 * size * normal(n) * real, size * (0.5 + uniform(n)) * real
        del size, real
        if case["bits"] == 32:
            s["m"], s["v"] = m, r * r
        else:
            s["m"], s["m_scale"] = _to8(m)
            s["v"], s["v_scale"] = _to8(r, E4M3_TINY)  # a second moment that is not zero is not stored as zero
        if case["master"]:
            s["w"] = s["p"].float() + 1e-4 * normal(n) * s["p"].float().abs()
            s["p"] = s["w"].to(io)
        s["tensors"] = {k: _views(s[k], case, begins, BLOCK if "scale" in k else 1) for k in ("p", "g", "m", "v", "w", "m_scale", "v_scale") if k in s}
        return s
    B, L, hk, hv, dk, dv = (case[k] for k in ("B", "L", "hk", "hv", "dk", "dv"))
    unit = torch.nn.functional.normalize
    s = dict(case=case, scale=dk ** -0.5, lengths=None, s0=None)
    s["q"] = unit(normal(B, L, hk, dk), dim=-1).to(io)
    s["k"] = unit(normal(B, L, hk, dk), dim=-1).to(io)
    s["v"] = normal(B, L, hv, dv).to(io)
    s["g"] = -torch.nn.functional.softplus(normal(B, L, hv) - 3.0).to(io)
    s["beta"] = torch.sigmoid(normal(B, L, hv)).to(io)
    if case["ragged"]:
        n = (uniform(B) * (L + 1)).int().clamp(max=L)
        n[0] = L
        if B > 2:
            n[1], n[2] = 0, 1
        s["lengths"] = n
    if case["kind"] == "steps" or case["state"]:
        s["s0"] = normal(B, hv, dk, dv) * dk ** -0.5
    if case["kind"] == "train":
        s["do"] = normal(B, L, hv, dv).to(io)
        s["ds"] = normal(B, hv, dk, dv) if case["state"] else None
        for k in ("q", "k", "v", "g", "beta", "s0"):
            if s[k] is not None:
                s[k].requires_grad_(True)
    if case["kind"] == "steps":
        s["o"] = torch.empty_like(s["v"])
    return s


def _to8(x, floor=0.0):
    """Blocks of 256 values as float8 e4m3 and their scales; a positive value is stored as no less than `floor`."""
    x = x.view(-1, BLOCK)
    top = x.abs().amax(1)
    scale = top / E4M3_MAX
    inverse = torch.where(top > 0, E4M3_MAX / top, torch.zeros_like(top)).clamp(max=torch.finfo(torch.float32).max)
    y = x * inverse[:, None]
    y = torch.where((x > 0) & (y < floor), torch.full_like(y, floor), y)
    return y.to(torch.float8_e4m3fn).view(-1), scale


def run(state):
    kind = state["case"]["kind"]
    if kind == "adamw":
        return _own_adamw(state) if own else _plain_adamw(state)
    if kind == "steps":
        return _own_steps(state) if own else _plain_steps(state)
    if own:
        from paper_2406_12580_gb300.delta import gated_delta_rule as rule
    else:
        rule = _plain_rule
    names = [k for k in ("q", "k", "v", "g", "beta", "s0") if state[k] is not None]
    if kind == "prefill":
        with torch.no_grad():
            o, s = rule(*[state[k] for k in ("q", "k", "v", "g", "beta")], scale=state["scale"], s0=state["s0"], lengths=state["lengths"], with_state=True)
        return {"o": o, "s": s}
    o, s = rule(*[state[k] for k in ("q", "k", "v", "g", "beta")], scale=state["scale"], s0=state["s0"], lengths=state["lengths"], with_state=state["ds"] is not None)
    outs, grads = ([o], [state["do"]]) if state["ds"] is None else ([o, s], [state["do"], state["ds"]])
    d = torch.autograd.grad(outs, [state[k] for k in names], grads)
    return {"o": o.detach(), **({} if s is None else {"s": s.detach()}), **{"d" + k: x for k, x in zip(names, d)}}


# the framework's calls


def _own_steps(state):
    from paper_2406_12580_gb300 import BLR_BF16, BLR_F32, GDRDesc, blr_gdr_steps
    c = state["case"]
    desc = GDRDesc(c["B"], c["L"], c["hk"], c["hv"], c["dk"], c["dv"], io=BLR_BF16 if c["io"] == "bf16" else BLR_F32, scale=state["scale"])
    blr_gdr_steps(desc, BLR_F32, state["s0"], state["q"], state["k"], state["v"], state["g"], state["beta"], state["s0"], state["o"])
    return {"o": state["o"], "s": state["s0"]}


def _own_adamw(state):
    from paper_2406_12580_gb300 import blr_adamw_step
    state["step"] += 1
    t = state["tensors"]
    blr_adamw_step(t["p"], t["g"], t["m"], t["v"], masters=t.get("w"), m_scales=t.get("m_scale"), v_scales=t.get("v_scale"), step=state["step"], **HYPER)
    return {k: state[k] for k in ("p", "w", "m", "v", "m_scale", "v_scale") if k in state}


HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)

# the plain forms, in 32 bits


def _plain_steps(state):
    q, k, v, g, beta = (state[x].float() for x in ("q", "k", "v", "g", "beta"))
    group = v.shape[2] // q.shape[2]
    q, k = (x.repeat_interleave(group, 2) for x in (q, k))
    S, out = state["s0"], []
    for t in range(v.shape[1]):
        S = S * torch.exp(g[:, t, :, None, None])
        u = beta[:, t, :, None] * (v[:, t] - (k[:, t, :, None, :] @ S).squeeze(-2))
        S = S + k[:, t, :, :, None] * u[:, :, None, :]
        out.append((q[:, t, :, None, :] @ S).squeeze(-2) * state["scale"])
    state["s0"].copy_(S)
    state["o"].copy_(torch.stack(out, 1))
    return {"o": state["o"], "s": state["s0"]}


def _inverse(A):
    """(I + A)^-1 of strictly lower triangular blocks, by halves: 1 x 1 blocks, joined to 2 x 2, 4 x 4, ..."""
    n, s = A.shape[-1], 1
    T = torch.ones(*A.shape[:-2], n, 1, 1, dtype=A.dtype, device=A.device)
    while s < n:
        i = torch.arange(n // (2 * s), device=A.device)
        low = A.view(*A.shape[:-2], n // (2 * s), 2, s, n // (2 * s), 2, s).movedim((-6, -3), (0, 1))[i, i][..., 1, :, 0, :].movedim(0, -3)
        a, b = T[..., 0::2, :, :], T[..., 1::2, :, :]
        T = torch.cat([torch.cat([a, torch.zeros_like(a)], -1), torch.cat([-b @ low @ a, b], -1)], -2)
        s *= 2
    return T.squeeze(-3)


def _plain_rule(q, k, v, g, beta, scale, s0=None, lengths=None, with_state=False):
    """Chunks of 64 steps: what does not hang on the state for all chunks at once, then the states from chunk to chunk."""
    B, L, hk, dk = q.shape
    hv, dv = v.shape[2:]
    io = v.dtype
    group, n = hv // hk, -(-L // CHUNK)
    q, k, v, g, beta = (x.float() for x in (q, k, v, g, beta))
    if lengths is not None:
        real = torch.arange(L, device=q.device)[None, :] >= L - lengths[:, None]
        q, k, v, g, beta = (torch.where(real.view(B, L, *[1] * (x.dim() - 2)), x, torch.zeros_like(x)) for x in (q, k, v, g, beta))
    q, k = (x.repeat_interleave(group, 2) for x in (q, k))

    def chunks(x):  # (B, L, H, ...) -> (B, H, n, CHUNK, ...)
        x = torch.nn.functional.pad(x, [0, 0] * (x.dim() - 2) + [0, n * CHUNK - L])
        return x.view(B, n, CHUNK, *x.shape[2:]).movedim(3, 1)

    q, k, v, g, beta = chunks(q), chunks(k), chunks(v), chunks(g), chunks(beta)
    G = g.cumsum(-1)
    lower = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=q.device).tril()
    decay = torch.exp((G[..., :, None] - G[..., None, :]).masked_fill(~lower, -math.inf))
    kt = k.transpose(-1, -2)
    T = _inverse((beta[..., None] * decay * (k @ kt)).tril(-1))
    up, end = torch.exp(G)[..., None], torch.exp(G[..., -1:] - G)[..., None]
    W, U0 = T @ (beta[..., None] * up * k), T @ (beta[..., None] * v)
    last, kend = torch.exp(G[..., -1])[..., None, None], (end * k).transpose(-1, -2)
    S = torch.zeros(B, hv, dk, dv, device=q.device) if s0 is None else s0
    before, us = [], []
    for c in range(n):
        before.append(S)
        us.append(U0[:, :, c] - W[:, :, c] @ S)
        S = last[:, :, c] * S + kend[:, :, c] @ us[-1]
    U = torch.stack(us, 2)
    o = scale * (up * (q @ torch.stack(before, 2)) + (decay * (q @ kt)) @ U)
    o = o.movedim(1, 3).reshape(B, n * CHUNK, hv, dv)[:, :L].to(io)
    return o, S if with_state else None


def _from8(x, scale):
    return x.float() * scale.repeat_interleave(BLOCK)


def _plain_adamw(state):
    h, case = HYPER, state["case"]
    state["step"] += 1
    g = state["g"].float()
    w = state["w"] if case["master"] else state["p"].float()
    if case["bits"] == 32:
        m, v = state["m"], state["v"]
    else:
        m, v = _from8(state["m"], state["m_scale"]), _from8(state["v"], state["v_scale"])
        v = v * v
    m = m * h["beta1"] + g * (1 - h["beta1"])
    v = v * h["beta2"] + g * g * (1 - h["beta2"])
    root = torch.sqrt(v)
    denominator = root * (1 / math.sqrt(1 - h["beta2"] ** state["step"])) + h["eps"]
    w = w * (1 - h["lr"] * h["weight_decay"]) - m / denominator * (h["lr"] / (1 - h["beta1"] ** state["step"]))
    if case["bits"] == 32:
        state["m"].copy_(m)
        state["v"].copy_(v)
    else:
        for name, x, floor in (("m", m, 0.0), ("v", root, E4M3_TINY)):
            values, scale = _to8(x, floor)
            state[name].copy_(values)
            state[name + "_scale"].copy_(scale)
    state["p"].copy_(w)
    if case["master"]:
        state["w"].copy_(w)
    return {k: state[k] for k in ("p", "w", "m", "v", "m_scale", "v_scale") if k in state}


# what an operator cannot do without


def work(case):
    e = 2 if case["io"] == "bf16" else 4
    if case["kind"] == "adamw":
        n = sum(math.prod(s) for s in _shapes(case))
        state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        return {"bytes": n * (3 * e - (e if case["master"] else 0) + state + (8 if case["master"] else 0)), "flops": 15 * n}
    B, L, hk, hv, dk, dv = (case[k] for k in ("B", "L", "hk", "hv", "dk", "dv"))
    tokens = B * L
    if case["ragged"]:
        tokens = L + (1 if B > 2 else 0) + max(0, B - (3 if B > 2 else 1)) * L / 2  # what the lengths come to on average
    keys, values, gates, states = 2 * tokens * hk * dk * e, tokens * hv * dv * e, 2 * tokens * hv * e, B * hv * dk * dv * 4
    has = case["kind"] == "steps" or case["state"]
    size, flops = keys + 2 * values + gates + (2 * states if has else 0), 7 * tokens * hv * dk * dv
    if case["kind"] == "train":
        size += values + keys + values + gates + (2 * states if has else 0)
        flops += 15 * tokens * hv * dk * dv
    if case["kind"] == "prefill" and not case["state"]:
        size += states
    return {"bytes": size, "flops": flops}


# the definitions in 64 bits


def exact(case, seed):
    state = prepare(case, seed)
    return _exact_adamw(state) if case["kind"] == "adamw" else _exact_gdr(state)


def _exact_adamw(state):
    """Tensor by tensor, from the definition."""
    case, t = state["case"], state["tensors"]
    step = state["step"] + 1
    b1, b2 = HYPER["beta1"], HYPER["beta2"]
    out = {k: torch.zeros(state[k].shape, dtype=torch.float64, device="cuda") for k in ("p", "w", "m", "v", "m_scale", "v_scale") if k in state}
    begins, _ = _places(case)
    for i, b in enumerate(begins):
        p = t["w" if case["master"] else "p"][i].double().flatten()
        g, n = t["g"][i].double().flatten(), t["g"][i].numel()
        if case["bits"] == 32:
            m, v = t["m"][i].double().flatten(), t["v"][i].double().flatten()
        else:
            where = torch.arange(n, device="cuda") // BLOCK
            m = t["m"][i].flatten().float().double() * t["m_scale"][i].double()[where]
            v = (t["v"][i].flatten().float().double() * t["v_scale"][i].double()[where]) ** 2
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g ** 2
        p = p - HYPER["lr"] * HYPER["weight_decay"] * p
        p = p - HYPER["lr"] * (m / (1 - b1 ** step)) / ((v / (1 - b2 ** step)).sqrt() + HYPER["eps"])
        out["p"][b:b + n] = p
        if case["master"]:
            out["w"][b:b + n] = p
        if case["bits"] == 32:
            out["m"][b:b + n], out["v"][b:b + n] = m, v
            continue
        for name, x, floor in (("m", m, 0.0), ("v", v.sqrt(), E4M3_TINY)):
            blocks = -(-n // BLOCK)
            top = torch.zeros(blocks, dtype=torch.float64, device="cuda").scatter_reduce(0, where, x.abs(), "amax")
            code = x / (top / E4M3_MAX).clamp(min=1e-300)[where]
            code = torch.where(x > 0, code.clamp(min=floor), code)
            out[name][b:b + n] = code.float().to(torch.float8_e4m3fn).double()
            out[name + "_scale"][b // BLOCK:b // BLOCK + blocks] = top / E4M3_MAX
    return out


def _exact_gdr(state):
    """Step by step; the gradients by the reverse recurrence over stretches whose states are computed again."""
    case, scale = state["case"], state["scale"]
    B, L, hk, hv, dk, dv = (case[k] for k in ("B", "L", "hk", "hv", "dk", "dv"))
    q, k, v, g, beta = (state[x].detach().double() for x in ("q", "k", "v", "g", "beta"))
    if state["lengths"] is not None:
        pad = torch.arange(L, device="cuda")[None, :] < L - state["lengths"][:, None]
        for x in (q, k, v, g, beta):
            x[pad] = 0.0
    q, k = (x.repeat_interleave(hv // hk, 2).transpose(0, 1).contiguous() for x in (q, k))
    v, g, beta = (x.transpose(0, 1).contiguous() for x in (v, g, beta))
    a = g.exp()

    def step(S, t):
        D = S * a[t, :, :, None, None]
        rest = v[t] - torch.einsum("bhk,bhkv->bhv", k[t], D)
        u = rest * beta[t, :, :, None]
        return D, rest, u, D + k[t, :, :, :, None] * u[:, :, None, :]

    S = torch.zeros(B, hv, dk, dv, dtype=torch.float64, device="cuda")
    if state["s0"] is not None:
        S = S + state["s0"].detach().double()
    train = case["kind"] == "train"
    stretch = max(1, min(L, int(6e9 / (3 * 8 * S.numel()))))
    stretch = min(stretch, max(32, math.isqrt(L)))
    o, kept = torch.zeros(L, B, hv, dv, dtype=torch.float64, device="cuda"), []
    for t in range(L):
        if train and t % stretch == 0:
            kept.append(S)
        S = step(S, t)[3]
        o[t] = scale * torch.einsum("bhk,bhkv->bhv", q[t], S)
    out = {"o": o.transpose(0, 1)}
    if case["kind"] == "steps" or case["kind"] == "prefill" or case["state"]:
        out["s"] = S
    if not train:
        return out
    do = state["do"].double().transpose(0, 1)
    if state["lengths"] is not None:
        do = torch.where(pad.t()[:, :, None, None], torch.zeros_like(do), do)
    dS = torch.zeros_like(S) if state["ds"] is None else state["ds"].double()
    dq, dk_, dv_, dg, db = (torch.zeros_like(x) for x in (q, k, v, g, beta))
    for c in range(len(kept) - 1, -1, -1):
        S, seen = kept.pop(), []
        for t in range(c * stretch, min(L, (c + 1) * stretch)):
            D, rest, u, S = step(S, t)
            seen.append((t, D, rest, u, S))
        while seen:
            t, D, rest, u, S = seen.pop()
            dq[t] = scale * torch.einsum("bhkv,bhv->bhk", S, do[t])
            dS = dS + scale * q[t, :, :, :, None] * do[t, :, :, None, :]
            du = torch.einsum("bhk,bhkv->bhv", k[t], dS)
            drest = du * beta[t, :, :, None]
            db[t] = (du * rest).sum(-1)
            dv_[t] = drest
            dk_[t] = torch.einsum("bhkv,bhv->bhk", dS, u) - torch.einsum("bhkv,bhv->bhk", D, drest)
            dD = dS - k[t, :, :, :, None] * drest[:, :, None, :]
            dg[t] = (dD * D).sum((-1, -2))
            dS = dD * a[t, :, :, None, None]
    if state["lengths"] is not None:
        for x in (dq, dk_, dv_, dg, db):
            x[pad.t()] = 0.0
    dq, dk_ = (x.transpose(0, 1).view(B, L, hk, hv // hk, dk).sum(3) for x in (dq, dk_))
    out.update(dq=dq, dk=dk_, dv=dv_.transpose(0, 1), dg=dg.transpose(0, 1), dbeta=db.transpose(0, 1))
    if state["s0"] is not None:
        out["ds0"] = dS
    return out
