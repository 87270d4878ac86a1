"""Inputs and a float64 statement of the gated delta rule, step by step with torch's autograd: what the
kernels are checked against. Shares no code with them."""
import torch


def make(B, L, Hk, Hv, Dk, Dv, dtype, seed, state=False, lengths=None, decay=(0.001, 0.3), device="cpu"):
    gen = torch.Generator().manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)  # noqa: E731
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
    lo, hi = decay
    d = dict(q=unit(normal(B, L, Hk, Dk)), k=unit(normal(B, L, Hk, Dk)), v=normal(B, L, Hv, Dv),
             g=-(lo + (hi - lo) * torch.rand(B, L, Hv, generator=gen, dtype=torch.float64)),
             beta=torch.sigmoid(normal(B, L, Hv)), do=normal(B, L, Hv, Dv))
    d = {k: x.to(dtype).to(device) for k, x in d.items()}
    d["s0"] = (normal(B, Hv, Dk, Dv) * Dk ** -0.5).float().to(device) if state else None
    d["ds"] = normal(B, Hv, Dk, Dv).float().to(device) if state else None
    d["lengths"] = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=device)
    d["scale"] = Dk ** -0.5
    return d


def reference(d, backward=True):
    """{name: float64 tensor}: o, s and the gradients, each row over its own steps."""
    leaf = {k: d[k].detach().double().cpu().requires_grad_(True) for k in ("q", "k", "v", "g", "beta")}
    B, L, Hk, Dk = leaf["q"].shape
    Hv, Dv = leaf["v"].shape[2:]
    s0 = torch.zeros(B, Hv, Dk, Dv, dtype=torch.float64) if d["s0"] is None else d["s0"].double().cpu()
    leaf["s0"] = s0.detach().clone().requires_grad_(True)
    group, outs, lasts = Hv // Hk, [], []
    for b in range(B):
        n = L if d["lengths"] is None else min(max(int(d["lengths"][b]), 0), L)
        S, rows = leaf["s0"][b], [torch.zeros(L - n, Hv, Dv, dtype=torch.float64)]
        for t in range(L - n, L):
            q, k = (leaf[x][b, t].repeat_interleave(group, 0) for x in ("q", "k"))
            S = S * torch.exp(leaf["g"][b, t].clamp(min=-120.0))[:, None, None]
            u = leaf["beta"][b, t][:, None] * (leaf["v"][b, t] - torch.einsum("hk,hkv->hv", k, S))
            S = S + k[:, :, None] * u[:, None, :]
            rows.append(d["scale"] * torch.einsum("hk,hkv->hv", q, S)[None])
        outs.append(torch.cat(rows))
        lasts.append(S)
    o, s = torch.stack(outs), torch.stack(lasts)
    out = {"o": o.detach(), "s": s.detach()}
    if backward:
        pad = torch.zeros(B, L, dtype=torch.bool)
        if d["lengths"] is not None:
            pad = torch.arange(L)[None, :] < L - d["lengths"].cpu().clamp(0, L)[:, None]
        do = torch.where(pad[:, :, None, None], torch.zeros((), dtype=torch.float64), d["do"].double().cpu())
        loss = (o * do).sum()
        if d["ds"] is not None:
            loss = loss + (s * d["ds"].double().cpu()).sum()
        names = ["q", "k", "v", "g", "beta", "s0"]
        grads = torch.autograd.grad(loss, [leaf[x] for x in names], allow_unused=True)
        out.update({"d" + n: torch.zeros_like(leaf[n]) if x is None else x for n, x in zip(names, grads)})
    return out


def off(got, want):
    """2-norm of the difference over the 2-norm of what is wanted, as float32 can hold it."""
    got, want = got.detach().double().cpu(), want.float().double()
    assert got.shape == want.shape and torch.isfinite(got).all()
    norm = float(want.norm())
    return float((got - want).norm()) / norm if norm else float(got.norm())
