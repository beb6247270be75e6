"""CPU tests of the operators' binding: operands whose memory is not what the kernels take it for are refused before the
library is called (a recorder, as in test_ops_devices)."""
import pytest
import torch

from tests.test_ops_devices import CALL, _bwd, _fwd, _on, _record, _tensors, library  # noqa: F401

A = pytest.importorskip("paper_2504_13850_amd.api")


@pytest.mark.parametrize("dtype", [torch.int32, torch.bfloat16, torch.float64])
def test_lse_of_another_type(library, dtype):  # noqa: F811
    x, a = _record()
    y = _tensors(CALL, 0)
    y["lse"] = _on(0, torch.zeros((2, 4), dtype=dtype))
    for call in (_fwd, _bwd):
        with pytest.raises(A.FoError):
            call(a, x, y)
    assert not library.calls
