"""Errors that were there before a call of an operator."""
import pytest
import torch
from test_gpu_operators import DEV, _ops

pytestmark = pytest.mark.gpu


def test_an_error_left_before_a_call_is_not_the_calls():
    from paper_2502_04557_amd import binding
    lib = binding.load_library()
    logits = torch.randn(4, 8, device=DEV)
    ids, w = torch.full((4, 2), -7, dtype=torch.int32, device=DEV), torch.empty(4, 2, device=DEV)
    want = _ops().route(logits, 2)
    cfg = _ops()._route_cfg(8, 2, "softmax", 1, 1, "max", True, 0, 1.0)
    torch.cuda.synchronize()
    assert lib.hipSetDevice(1 << 20) != 0                 # (refused on the host: there is no such device)
    rc = lib.sprinter_route(cfg[1], logits.data_ptr(), 8, None, 4, ids.data_ptr(), w.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert rc == 0, lib.sprinter_last_error(None)
    assert torch.equal(ids, want[0]) and torch.equal(w, want[1])
