"""The 8-bit operators where another device than that of their tensors is current.  One GPU is enough: the entry points are told that the current device is another one."""
import pytest
import torch

import paper_2605_28657_amd as pa

pytestmark = pytest.mark.gpu


def _layer(x, residual, weight, up, down):
    q, s, h = pa.rms_norm_fp8(x, weight, residual=residual)
    gu = pa.matmul_fp8(q, s, *up)
    g, gs = pa.quantize_fp8(gu, gated=True)
    return [q.view(torch.uint8), s, h, gu, g.view(torch.uint8), gs, pa.matmul_fp8(g, gs, *down, fp32_sums=True), up[0].view(torch.uint8), up[1]]


def test_the_device_of_the_tensors_is_taken(monkeypatch):
    g = torch.Generator().manual_seed(1)
    normal = lambda *shape: torch.randn(shape, generator=g).bfloat16().to("cuda:0")      # noqa: E731
    x, r, w, up, down = normal(40, 320), normal(40, 320), torch.ones(320, device="cuda:0"), normal(1408, 320), normal(320, 704)
    run = lambda: _layer(x, r, w, pa.quantize_weights_fp8(up), pa.quantize_weights_fp8(down))      # noqa: E731
    want = run()
    torch.cuda.synchronize()
    entered = []
    device = torch.cuda.device

    class Recorded(device):
        def __enter__(self):
            entered.append(self.idx)
            return super().__enter__()

    side = torch.cuda.Stream("cuda:0")
    with torch.cuda.stream(side), monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        m.setattr(torch.cuda, "device", Recorded)
        got = run()
    side.synchronize()
    assert entered == [0] * 6                               # every launch with the tensors' device current
    assert all(torch.equal(a, b) for a, b in zip(got, want))
