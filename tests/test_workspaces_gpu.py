"""Workspaces that a caller brings to the backward passes: any type, on the GPU, contiguous, large enough."""
import pytest
import torch

from paper_1911_04477_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def calls():
    x, wg, wu = (torch.randn(s, device=DEV).bfloat16() for s in ((6, 32), (24, 32), (24, 32)))
    dh, w = torch.randn((6, 24), device=DEV).bfloat16(), torch.rand(32, device=DEV)
    saved = B.gated_ff_saved(6, 24, DEV)
    B.bnn_gated_ff(x, wg, wu, saved=saved)
    return ((B.gated_ff_backward_workspace_bytes(6, 32, 24),
             lambda ws: B.bnn_gated_ff_backward(x, wg, wu, saved, dh, workspace=ws)),
            (B.norm_gate_backward_workspace_bytes(6, 32, 0),
             lambda ws: tuple(B.bnn_norm_gate_backward(x, x, x, x, w_pre=w, workspace=ws).values())))


@pytest.mark.parametrize("direct", [True, False])
def test_workspaces(direct, monkeypatch):
    """Both by the calls from tensors and by those through ctypes' arguments."""
    cases = calls()
    if not direct:
        class Declines:
            def __getattr__(self, name):
                return lambda *args: None

        monkeypatch.setattr(B, "_t", Declines)
    for nbytes, call in cases:
        words = -(-nbytes // 4)
        want = call(None)
        for ws in (torch.empty(nbytes, dtype=torch.uint8, device=DEV), torch.empty(words, device=DEV), torch.empty((2, words), device=DEV)):
            assert all(torch.equal(a, b) for a, b in zip(call(ws), want))
        with pytest.raises(TypeError, match="workspace"):
            call(torch.empty(nbytes, dtype=torch.uint8))
        with pytest.raises(ValueError, match="workspace"):
            call(torch.empty(4 * nbytes, dtype=torch.uint8, device=DEV)[::2])
        with pytest.raises(B.BnnError):
            call(torch.empty(nbytes - 1, dtype=torch.uint8, device=DEV))
