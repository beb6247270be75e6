"""CPU tests of the operators' binding: operands whose memory is not what the kernels take it for are refused before the
library is called (a recorder, as in test_ops_devices)."""
import pytest
import torch

from tests.test_ops_devices import CALL, DROP, _bwd, _drop, _drop_back, _fwd, _on, _record, _tensors, library  # noqa: F401

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


def test_expanded_tensors(library):  # noqa: F811
    """One element repeated by a stride of zero stands for less memory than its shape says."""
    x, a = _record()
    y = _tensors(CALL, 0)
    y["workspace"] = _on(0, torch.zeros(1, dtype=torch.uint8).expand(1 << 20))
    for call in (_fwd, _bwd):
        with pytest.raises(A.FoError):
            call(a, x, y)
    for name, t in (("workspace", torch.zeros(1, dtype=torch.uint8).expand(1 << 20)),
                    ("dbias", torch.zeros((1, 1), dtype=torch.bfloat16).expand(8, 1)),
                    ("bias", torch.zeros((1, 1), dtype=torch.bfloat16).expand(8, 1))):
        with pytest.raises(A.FoError):
            (_drop if name == "bias" else _drop_back)({**_tensors(DROP, 0), name: _on(0, t)})
    assert not library.calls
