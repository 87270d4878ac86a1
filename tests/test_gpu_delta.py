"""GPU: the gated delta rule (whole sequences with gradients, and recurrent steps) against a float64
statement of it, at the lengths, masks, heads, strides and types where chunked kernels go wrong."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU machines, but never run there
    pytest.skip("no CUDA device", allow_module_level=True)

from delta_common import make, off, reference  # noqa: E402
from paper_2406_12580_gb300 import (BLR_BF16, BLR_F32, BLRError, GDRDesc, blr_gdr_fwd, blr_gdr_steps,  # noqa: E402
                                    blr_gdr_workspace_bytes)
from paper_2406_12580_gb300.delta import GatedDeltaLayer, gated_delta_rule  # noqa: E402

# Bounds on the 2-norm error over the 2-norm. Operands of two bfloat16 terms are off by at most 2^-18 of
# themselves, and at most about ten of them stand in a row behind one output: sqrt(20) 2^-18 = 1.7e-5
# (float32 outputs). A bfloat16 output adds its own rounding, 2^-8 / sqrt(3) = 2.3e-3 at most over the
# mantissa. Products of bfloat16 operands round about ten numbers in a row, but their errors average
# over the sums: twice the output's rounding is allowed.
EXACT, ROUNDED, COARSE = 2e-5, 2.3e-3, 4.6e-3

SHAPES = [  # B, L, Hk, Hv, Dk, Dv, lengths
    (1, 1, 1, 1, 64, 64, None),
    (2, 63, 1, 2, 64, 128, None),
    (1, 64, 2, 2, 128, 64, None),
    (3, 65, 1, 1, 128, 128, None),
    (2, 200, 2, 4, 64, 64, None),
    (1, 129, 1, 1, 64, 192, None),
    (1, 70, 1, 3, 128, 256, None),
    (5, 131, 1, 2, 64, 64, [0, 131, 1, 64, 77]),
    (3, 257, 2, 2, 128, 128, [300, -5, 65]),
    # one chunk a row: no states without BLR_GDR_STATE
    (7, 50, 2, 2, 64, 64, [50, 0, 1, 49, 17, 33, 50]),
    (3, 64, 1, 2, 128, 128, [64, 20, 0]),
    # few heads and long rows: cut into segments
    (1, 2700, 1, 1, 64, 64, None),
    (3, 2600, 1, 1, 64, 128, [0, 2600, 130]),
    (2, 3333, 1, 1, 128, 64, [1111, 3333]),
]


def run(d, with_state):
    leaves = [d[n] for n in ("q", "k", "v", "g", "beta", "s0") if d[n] is not None]
    for x in leaves:
        x.requires_grad_(True)
    o, s = gated_delta_rule(*(d[n] for n in ("q", "k", "v", "g", "beta")), scale=d["scale"], s0=d["s0"],
                            lengths=d["lengths"], with_state=with_state)
    outs, grads = ([o, s], [d["do"], d["ds"]]) if d["ds"] is not None else ([o], [d["do"]])
    got = torch.autograd.grad(outs, leaves, grads)
    names = [n for n in ("q", "k", "v", "g", "beta", "s0") if d[n] is not None]
    return {"o": o, "s": s, **{"d" + n: x for n, x in zip(names, got)}}


@pytest.mark.parametrize("kind", ["f32", "f32_state", "bf16", "bf16_state"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward_and_gradients(shape, kind):
    *sizes, lengths = shape
    dtype = torch.float32 if kind.startswith("f32") else torch.bfloat16
    state = kind.endswith("state")
    d = make(*sizes, dtype, seed=3 + len(kind), state=state, lengths=lengths, device="cuda")
    if lengths is not None:  # the padding is not read
        pad = torch.arange(sizes[1], device="cuda")[None, :] < sizes[1] - d["lengths"].clamp(0, sizes[1])[:, None]
        want = reference(d)
        for n in ("q", "k", "v", "g", "beta", "do"):
            d[n][pad] = float("nan")
    else:
        want = reference(d)
    got = run(d, state)
    for n, x in got.items():
        if x is None:
            continue
        bound = EXACT if x.dtype == torch.float32 else COARSE
        if state and x.dtype == torch.bfloat16:
            # a few large values can round worse than the mean: the reference's own rounding, and what the
            # 2e-5 before it turns into where a value lies that near a boundary, sqrt(2e-5 2^-8)
            bound = off(want[n].bfloat16(), want[n]) + 3e-4
        assert off(x, want[n]) <= bound, (n, off(x, want[n]))
        if lengths is not None and n not in ("s", "ds0"):
            assert not x.detach()[pad].any(), n


@pytest.mark.parametrize("decay", [(0.0, 0.0), (5.0, 30.0), (90.0, 400.0), (0.0, 60.0)], ids=str)
def test_decays_from_none_to_all(decay):
    d = make(2, 150, 1, 2, 64, 64, torch.float32, seed=8, state=True, decay=decay, device="cuda")
    want, got = reference(d), run(d, True)
    for n in ("o", "s", "dq", "dk", "dv", "dbeta", "ds0"):
        assert off(got[n], want[n]) <= EXACT, n
    # the decay's gradient is a difference of sums: held against the size of what it is the difference of
    scale = float(want["dg"].norm()) + float(want["dbeta"].norm())
    assert float((got["dg"].double().cpu() - want["dg"]).norm()) <= EXACT * scale


def test_equal_keys():
    """One key at every step with full write strength: the chunk's triangular system is as stiff as it gets.
    The outputs are then sums of up to 64 u whose exact values cancel to one: sqrt(64) times the bound."""
    d = make(1, 130, 1, 1, 64, 64, torch.float32, seed=9, state=True, decay=(0.0, 0.001), device="cuda")
    d["k"][:] = d["k"][0, 0, 0].clone()
    d["beta"].fill_(1.0)
    want, got = reference(d), run(d, True)
    for n in ("o", "s", "dv", "dq", "ds0"):
        assert off(got[n], want[n]) <= 8 * EXACT, n


@pytest.mark.parametrize("name", ["q", "k", "v", "g", "beta", "s0"])
def test_gradients_against_differences(name):
    """<gradient, direction> against the float32 forward's central difference, whose error is h^2 of the
    third derivative (h^2 = 4e-4 of order-one terms) plus the forward's 2e-5 / h of its values."""
    d = make(2, 100, 1, 2, 64, 64, torch.float32, seed=10, state=True, device="cuda")
    got = run(d, True)
    x = d[name].detach()
    e = torch.randn(x.shape, generator=torch.Generator().manual_seed(1)).to("cuda") * got["d" + name].sign().abs()
    e = e * x.abs() if name == "g" else e * x.std()
    h, values = 0.02, []
    for s in (h, -h):
        c = {**{n: (t.detach() if torch.is_tensor(t) else t) for n, t in d.items()}, name: x + s * e}
        with torch.no_grad():
            o, sl = gated_delta_rule(*(c[n] for n in ("q", "k", "v", "g", "beta")), scale=c["scale"], s0=c["s0"],
                                     with_state=True)
        values.append(float((o.double() * d["do"].double()).sum() + (sl.double() * d["ds"].double()).sum()))
    slope = (values[0] - values[1]) / (2 * h)
    want = float((got["d" + name].double() * e.double()).sum())
    size = float((got["d" + name].double() * e.double()).norm()) + abs(want)
    assert abs(slope - want) <= 5e-3 * size, (slope, want)


def test_slices_of_wider_rows():
    """q, k and v as slices of one projection's output give what copies give, bit for bit."""
    B, L, H, D = 2, 90, 2, 64
    wide = torch.randn(B, L, 3 * H * D + 8, device="cuda", dtype=torch.bfloat16)
    q, k, v = (wide[..., i * H * D:(i + 1) * H * D].unflatten(-1, (H, D)) for i in range(3))
    q, k = q / 8, k / 8
    wide[..., :H * D], wide[..., H * D:2 * H * D] = q.flatten(-2), k.flatten(-2)
    q, k, v = (wide[..., i * H * D:(i + 1) * H * D].unflatten(-1, (H, D)) for i in range(3))
    g, beta = -torch.rand(B, L, H, device="cuda").bfloat16(), torch.rand(B, L, H, device="cuda").bfloat16()
    a, sa = gated_delta_rule(q, k, v, g, beta, with_state=True)
    b, sb = gated_delta_rule(q.contiguous(), k.contiguous(), v.contiguous(), g, beta, with_state=True)
    assert torch.equal(a, b) and torch.equal(sa, sb)
    odd = [t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for t in (q, k, v)]  # heads outside steps
    c, sc = gated_delta_rule(*odd, g, beta, with_state=True)
    assert torch.equal(a, c) and torch.equal(sa, sc)


def test_repeats_and_streams():
    """The same bits again, on another stream, and from a second backward of one forward."""
    d = make(2, 300, 1, 2, 128, 128, torch.bfloat16, seed=12, device="cuda")
    a = run(d, False)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        b = run(d, False)
    side.synchronize()
    for n in a:
        assert a[n] is None or torch.equal(a[n], b[n]), n
    o, _ = gated_delta_rule(*(d[n] for n in ("q", "k", "v", "g", "beta")), scale=d["scale"])
    x = torch.autograd.grad(o, [d["k"], d["g"]], d["do"], retain_graph=True)
    y = torch.autograd.grad(o, [d["k"], d["g"]], d["do"])
    assert all(torch.equal(i, j) for i, j in zip(x, y))


def test_captured_in_a_graph():
    d = make(2, 130, 1, 1, 64, 64, torch.bfloat16, seed=13, device="cuda")
    args = [d[n] for n in ("q", "k", "v", "g", "beta")]
    want, _ = gated_delta_rule(*args)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got, _ = gated_delta_rule(*args)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_split_sequences_carry_their_state():
    """Scanning [0, L) equals scanning [0, m) and then [m, L) from its state, m inside a chunk."""
    d = make(2, 200, 1, 2, 64, 64, torch.float32, seed=14, state=True, device="cuda")
    args = [d[n] for n in ("q", "k", "v", "g", "beta")]
    o, s = gated_delta_rule(*args, s0=d["s0"], with_state=True)
    _, half = gated_delta_rule(*(t[:, :77].contiguous() for t in args), s0=d["s0"], with_state=True)
    o2, s2 = gated_delta_rule(*(t[:, 77:].contiguous() for t in args), s0=half, with_state=True)
    assert off(o2, o[:, 77:].double().cpu()) <= 2 * EXACT and off(s2, s.double().cpu()) <= 2 * EXACT


STEPS = [(1, 1, 1, 2, 64, 64), (3, 4, 2, 2, 128, 64), (67, 2, 1, 1, 64, 128), (2, 9, 2, 4, 128, 256)]


@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("state", [BLR_F32, BLR_BF16])
@pytest.mark.parametrize("shape", STEPS, ids=str)
def test_steps(shape, io, state):
    d = make(*shape, io, seed=15, state=True, device="cuda")
    if state == BLR_BF16:
        d["s0"] = d["s0"].bfloat16()
    want = reference(d, backward=False)
    B, K, Hk, Hv, Dk, Dv = shape
    desc = GDRDesc(*shape, io=BLR_F32 if io == torch.float32 else BLR_BF16, scale=d["scale"])
    s, o = torch.empty_like(d["s0"]), torch.empty_like(d["v"])
    args = [d[n] for n in ("q", "k", "v", "g", "beta")]
    blr_gdr_steps(desc, state, d["s0"], *args, s, o)
    # float32 sums of at most 128 products: 2^-24 sqrt(128) a step, 9 steps
    assert off(o, want["o"]) <= (1e-5 if io == torch.float32 else ROUNDED)
    assert off(s, want["s"]) <= (1e-5 if state == BLR_F32 else ROUNDED)
    kept = d["s0"].clone()
    blr_gdr_steps(desc, state, d["s0"], *args, d["s0"], None)  # in place, without outputs
    assert torch.equal(d["s0"], s)
    none = GDRDesc(B, 0, Hk, Hv, Dk, Dv, io=desc.io, scale=1.0)
    blr_gdr_steps(none, state, kept, None, None, None, None, None, s, None)
    assert torch.equal(kept, s)
    blr_gdr_steps(none, state, None, None, None, None, None, None, s, None)
    assert not s.any()


def test_empty_sequences():
    d = make(2, 0, 1, 1, 64, 64, torch.float32, seed=16, state=True, device="cuda")
    o, s = gated_delta_rule(*(d[n] for n in ("q", "k", "v", "g", "beta")), s0=d["s0"], with_state=True)
    assert o.shape == (2, 0, 1, 64) and torch.equal(s, d["s0"])


def test_offsets_past_32_bits():
    """A batch whose q, k, v and o hold more than 2^31 values each: the last row equals the row alone."""
    B, L, H, D = 66, 65536, 4, 128
    if torch.cuda.get_device_properties(0).total_memory < 120 << 30:
        pytest.skip("needs 120 GB")
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(B, L, H, D, dtype=torch.bfloat16, device="cuda")
    x[:1].normal_(generator=gen)
    x[:1] /= 11.0
    x[-1:] = x[:1]
    g, beta = torch.full((B, L, H), -0.05, device="cuda").bfloat16(), torch.full((B, L, H), 0.5, device="cuda").bfloat16()
    lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
    lengths[0] = lengths[-1] = L
    lengths[1:-1] = 100
    x[1:-1, L - 100:] = x[:1, :100]
    o, _ = gated_delta_rule(x, x, x, g, beta, lengths=lengths)
    assert torch.equal(o[-1], o[0]) and o[0].any()
    assert not o[1, :L - 100].any() and torch.equal(o[1], o[-2])


def test_layer_steps_follow_its_sequences():
    """The layer's steps on kept states give its sequence form's outputs."""
    torch.manual_seed(0)
    layer = GatedDeltaLayer(32, heads=2, key_heads=1, device="cuda")
    x = torch.randn(3, 70, 32, device="cuda")
    with torch.no_grad():
        y, s = layer(x, with_state=True)
        states = torch.zeros_like(s)
        first, rest = layer.step(x[:, :1], states), layer.step(x[:, 1:], states)
    assert off(torch.cat([first, rest], 1), y.double().cpu()) <= 1e-4 and off(states, s.double().cpu()) <= 1e-4
    y = layer(x, lengths=torch.tensor([70, 0, 5], dtype=torch.int32, device="cuda"))
    y.square().sum().backward()
    assert all(torch.isfinite(p.grad).all() for p in layer.parameters())


def test_refusals():
    d = make(1, 64, 1, 1, 64, 64, torch.float32, seed=17, device="cuda")
    args = [d[n] for n in ("q", "k", "v", "g", "beta")]
    with pytest.raises(TypeError):
        gated_delta_rule(args[0].bfloat16(), *args[1:])
    with pytest.raises(ValueError):
        gated_delta_rule(*args, s0=torch.zeros(1, 1, 64, 32, device="cuda"))
    with pytest.raises(ValueError):
        gated_delta_rule(*args, lengths=torch.ones(1, device="cuda"))
    with pytest.raises(BLRError):
        gated_delta_rule(args[0][..., :32], args[1][..., :32], *args[2:])
    desc = GDRDesc(1, 64, 1, 1, 64, 64)
    o, s = torch.empty_like(d["v"]), torch.empty(1, 1, 64, 64, device="cuda")
    ws = torch.empty(blr_gdr_workspace_bytes(desc, 2), dtype=torch.uint8, device="cuda")
    with pytest.raises(BLRError):  # a state without its flag
        blr_gdr_fwd(desc, 0, None, *args, s, o, None, ws)
    with pytest.raises(BLRError):  # a workspace too small
        blr_gdr_fwd(desc, 2, None, *args, None, o, None, ws[:-16])
    assert ctypes.sizeof(desc) == 80


def test_no_second_derivative():
    d = make(1, 20, 1, 1, 64, 64, torch.float32, seed=18, device="cuda")
    q = d["q"].requires_grad_(True)
    o, _ = gated_delta_rule(q, *(d[n] for n in ("k", "v", "g", "beta")))
    with pytest.raises(RuntimeError):
        torch.autograd.grad(o.sum(), q, create_graph=True)


def test_not_a_number_is_not_hidden():
    """A NaN among the gates or values shows in what comes after it in its row, and in no other row."""
    for name in ("g", "beta", "v"):
        d = make(2, 100, 1, 1, 64, 64, torch.bfloat16, seed=19, device="cuda")
        d[name][1, 40] = float("nan")
        o, _ = gated_delta_rule(*(d[n] for n in ("q", "k", "v", "g", "beta")))
        assert torch.isfinite(o[0]).all() and torch.isnan(o[1, 40:]).any(-1).all()


def test_status_of_a_workspace():
    from paper_2406_12580_gb300 import BLR_OK, blr_gdr_status
    d = make(1, 100, 1, 1, 64, 64, torch.bfloat16, seed=20, device="cuda")
    desc = GDRDesc(1, 100, 1, 1, 64, 64, io=BLR_BF16)
    ws = torch.full((blr_gdr_workspace_bytes(desc, 0),), 255, dtype=torch.uint8, device="cuda")
    blr_gdr_fwd(desc, 0, None, *(d[n] for n in ("q", "k", "v", "g", "beta")), None, torch.empty_like(d["v"]), None, ws)
    assert blr_gdr_status(ws) == BLR_OK
