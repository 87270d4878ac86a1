"""GPU: the gated delta rule and the AdamW step together, as the next-item example uses them, and the optimizer."""
import copy

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU machines, but never run there
    pytest.skip("no CUDA device", allow_module_level=True)

from paper_2406_12580_gb300.next_item import serve, train  # noqa: E402
from paper_2406_12580_gb300.optim import AdamW  # noqa: E402


@pytest.mark.parametrize("bits", [32, 8])
def test_trains_and_serves(bits):
    """The rule of a walk shows after two items: the loss falls well below a uniform guess, log 101 = 4.6, and
    the served recommendations are the sequence form's (float32: products of at most 128 terms in two tf32
    terms each, through two layers)."""
    model, losses = train(steps=120, bits=bits)
    assert losses[0] > 3.5 and sum(losses[-10:]) / 10 < 0.5 * losses[0], (losses[0], losses[-1])
    hits, off = serve(model)
    assert off <= 1e-3 and hits > 0.2


def model_and_grads(dtype):
    torch.manual_seed(2)
    ps = [torch.nn.Parameter(torch.randn(*s, device="cuda").to(dtype)) for s in [(33, 7), (5,), (300,)]]
    grads = [[torch.randn_like(p) for p in ps] for _ in range(6)]
    return ps, grads


def walk(ps, opt, grads):
    for g in grads:
        for p, x in zip(ps, g):
            p.grad = x.clone()
        opt.step()


@pytest.mark.parametrize("dtype,bits,master", [(torch.float32, 32, False), (torch.float32, 8, False),
                                               (torch.bfloat16, 32, True), (torch.bfloat16, 8, True)], ids=str)
def test_optimizer_resumes_where_it_was_saved(dtype, bits, master):
    ps, grads = model_and_grads(dtype)
    opt = AdamW(ps, lr=1e-2, bits=bits, master=master)
    walk(ps, opt, grads[:3])
    saved, at = copy.deepcopy(opt.state_dict()), [p.detach().clone() for p in ps]
    walk(ps, opt, grads[3:])
    qs = [torch.nn.Parameter(x) for x in at]
    other = AdamW(qs, lr=1e-2, bits=bits, master=master)
    other.load_state_dict(saved)
    walk(qs, other, grads[3:])
    assert all(torch.equal(p, q) for p, q in zip(ps, qs))
    for p, q in zip(ps, qs):
        a, b = opt.state[p], other.state[q]
        assert all(a[n].dtype == b[n].dtype for n in a if torch.is_tensor(a[n]))


def test_optimizer_skips_what_has_no_gradient_and_scales():
    ps, grads = model_and_grads(torch.float32)
    opt = AdamW(ps, lr=1e-2)
    before = [p.detach().clone() for p in ps]
    ps[0].grad = grads[0][0].clone()
    opt.step(grad_scale=torch.zeros(1, device="cuda"))  # no gradient is left: only the weights' decay
    assert torch.allclose(ps[0], before[0] * (1 - 1e-4), rtol=1e-6) and torch.equal(ps[1], before[1])
    with pytest.raises(ValueError):
        AdamW(ps, bits=4)
