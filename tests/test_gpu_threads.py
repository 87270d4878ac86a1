"""GPU: calls from a thread that has made no CUDA call yet (as autograd's workers, whose memory comes from a cache)."""
import threading

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU machines, but never run there
    pytest.skip("no CUDA device", allow_module_level=True)

from delta_common import make  # noqa: E402
from paper_2406_12580_gb300 import (BLR_BF16, BLR_GDR_TRAIN, GDRDesc, blr_gdr_bwd, blr_gdr_fwd,  # noqa: E402
                                    blr_gdr_workspace_bytes)
from paper_2406_12580_gb300 import inputs as I  # noqa: E402
from paper_2406_12580_gb300.device import ScanBuffers  # noqa: E402


def in_new_thread(call):
    raised = []

    def body():
        try:
            call()
        except Exception as e:  # noqa: BLE001
            raised.append(e)

    t = threading.Thread(target=body)
    t.start()
    t.join()
    torch.cuda.synchronize()
    if raised:
        raise raised[0]


def test_gated_delta_rule():
    d = make(2, 100, 1, 1, 64, 64, torch.bfloat16, seed=31, device="cuda")
    args = [d[n].detach() for n in ("q", "k", "v", "g", "beta")]
    desc = GDRDesc(2, 100, 1, 1, 64, 64, io=BLR_BF16)
    ws = torch.empty(blr_gdr_workspace_bytes(desc, BLR_GDR_TRAIN), dtype=torch.uint8, device="cuda")
    outs = [[torch.empty_like(t) for t in (args[2], *args)] for _ in range(2)]
    stream = torch.cuda.current_stream()

    def fwd(o):
        blr_gdr_fwd(desc, BLR_GDR_TRAIN, None, *args, None, o[0], None, ws, stream=stream)

    def bwd(o):
        blr_gdr_bwd(desc, BLR_GDR_TRAIN, None, d["do"], None, *args, None, *o[1:], None, ws, stream=stream)

    fwd(outs[0])
    bwd(outs[0])
    in_new_thread(lambda: fwd(outs[1]))
    in_new_thread(lambda: bwd(outs[1]))
    for a, b in zip(*outs):
        assert torch.equal(a, b)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_scan(io):
    """One warp a chain: a fixed order of sums, so the outputs are the same bits."""
    inp = I.make_scan_inputs(I.ScanConfig("thread", B=256, L=50, D=64, io=io, seed=32))
    a, b = ScanBuffers.from_inputs(inp), ScanBuffers.from_inputs(inp)
    stream = torch.cuda.current_stream()
    a.fwd(stream)
    a.bwd(stream)
    in_new_thread(lambda: b.fwd(stream))
    in_new_thread(lambda: b.bwd(stream))
    for n in ("h", "h_last", "dx", "dgl", "dh0"):
        assert torch.equal(getattr(a, n), getattr(b, n)), n
