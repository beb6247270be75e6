"""CPU tests of the operators' binding: what is not on the GPU of the call is refused before the library is called.

Tensors in host memory stand in for those of a GPU by the device number that they give; the library behind the binding
is a recorder, so that a call that goes through can be told from one that is refused."""
import types

import pytest
import torch

A = pytest.importorskip("paper_2504_13850_amd.api")
BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


class _Gpu0(torch.Tensor):
    def get_device(self):
        return 0


class _Gpu1(torch.Tensor):
    def get_device(self):
        return 1


def _on(where, t):
    return t if where == "cpu" else t.as_subclass(_Gpu0 if where == 0 else _Gpu1)


class _Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append(name) or A.FO_OK


@pytest.fixture
def library(monkeypatch):
    rec = _Recorder()
    monkeypatch.setattr(A, "_lib", rec)
    return rec


STREAM = types.SimpleNamespace(cuda_stream=0, device_index=0)
RECORD = {"q": (BF16, 4, 2, 8), "k": (BF16, 6, 1, 8), "v": (BF16, 6, 1, 8), "out": (BF16, 4, 2, 8), "q_begin": (I32, 1),
          "q_end": (I32, 1), "k_begin": (I32, 1), "k_end": (I32, 1), "prefix": (I32, 1), "table": (BF16, 4, 2),
          "bucket": (I32, 5)}
CALL = {"lse": (F32, 2, 4), "dout": (BF16, 4, 2, 8), "dq": (BF16, 4, 2, 8), "dk": (BF16, 6, 1, 8), "dv": (BF16, 6, 1, 8),
        "dtable": (BF16, 4, 2), "workspace": (U8, 1024)}


def _tensors(spec, where, other=None):
    return {n: _on(where if other is None or n not in other else other[n], torch.zeros(s, dtype=dt))
            for n, (dt, *s) in spec.items()}


def _record(**at):
    x = _tensors(RECORD, 0, at)
    return x, A.make_attn(**x, max_q=4, max_k=4, mask=A.FO_ATTN_PREFIX)


def _fwd(a, x, y, stream=STREAM):
    A.fo_attn_fwd(a, x["q"], x["k"], x["v"], x["out"], y["lse"], y["workspace"], stream=stream)


def _bwd(a, x, y, stream=STREAM):
    A.fo_attn_bwd(a, x["q"], x["k"], x["v"], x["out"], y["lse"], y["dout"], y["dq"], y["dk"], y["dv"], y["dtable"],
                  y["workspace"], stream=stream)


def test_attention_on_one_gpu_goes_through(library):
    x, a = _record()
    y = _tensors(CALL, 0)
    _fwd(a, x, y)
    _bwd(a, x, y)
    assert library.calls == ["fo_attn_fwd", "fo_attn_bwd"]


@pytest.mark.parametrize("where", ["cpu", 1])
@pytest.mark.parametrize("name", list(RECORD))
def test_record_of_two_devices(where, name):
    with pytest.raises(A.FoError):
        _record(**{name: where})


def test_attention_in_host_memory(library):
    x = _tensors(RECORD, "cpu")
    a, y = A.make_attn(**x, max_q=4, max_k=4, mask=A.FO_ATTN_PREFIX), _tensors(CALL, "cpu")
    for call in (_fwd, _bwd):
        with pytest.raises(A.FoError):
            call(a, x, y)
    assert not library.calls


@pytest.mark.parametrize("where", ["cpu", 1])
@pytest.mark.parametrize("name", ["q", "k", "v", "out"] + list(CALL))
def test_attention_call_on_two_devices(library, where, name):
    x, a = _record()
    by_hand = A.fo_attn.from_buffer_copy(a)  # without what make_attn notes beside the record
    x.update({n: t for n, t in _tensors(RECORD, 0, {name: where}).items() if n == name})
    y = _tensors(CALL, 0, {name: where})
    for r in (a, by_hand):
        with pytest.raises(A.FoError):
            _bwd(r, x, y)
        if name in ("q", "k", "v", "out", "lse", "workspace"):
            with pytest.raises(A.FoError):
                _fwd(r, x, y)
    assert not library.calls


def test_stream_of_another_gpu(library, monkeypatch):
    x, a = _record()
    y = _tensors(CALL, 0)
    one = types.SimpleNamespace(cuda_stream=0, device_index=1)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for stream in (one, None):
        for call in (_fwd, _bwd):
            with pytest.raises(A.FoError):
                call(a, x, y, stream)
    z = _tensors({"x": (BF16, 4, 8), "y": (BF16, 4, 8)}, 0)
    with pytest.raises(A.FoError):
        A.fo_dropout_fwd(z["x"], z["y"], 0.1, 1, 1, stream=one)
    assert not library.calls
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    _fwd(a, x, y, None)
    assert library.calls == ["fo_attn_fwd"]


DROP = {"x": (BF16, 4, 8), "y": (BF16, 4, 8), "bias": (BF16, 8), "residual": (BF16, 4, 8), "dbias": (BF16, 8),
        "workspace": (U8, 1024)}


def _drop(x):
    A.fo_dropout_fwd(x["x"], x["y"], 0.1, 1, 1, bias=x["bias"], residual=x["residual"], stream=STREAM)


def _drop_back(x):
    A.fo_dropout_bwd(x["x"], x["y"], 0.1, 1, 1, dbias=x["dbias"], workspace=x["workspace"], stream=STREAM)


def test_dropout_on_one_gpu_goes_through(library):
    _drop(_tensors(DROP, 0))
    _drop_back(_tensors(DROP, 0))
    assert library.calls == ["fo_dropout_fwd", "fo_dropout_bwd"]


@pytest.mark.parametrize("where", ["cpu", 1])
@pytest.mark.parametrize("name", ["all"] + list(DROP))
def test_dropout_on_two_devices(library, where, name):
    x = _tensors(DROP, "cpu") if name == "all" else _tensors(DROP, 0, {name: where})
    if name not in ("dbias", "workspace"):
        with pytest.raises(A.FoError):
            _drop(x)
    if name not in ("bias", "residual"):
        with pytest.raises(A.FoError):
            _drop_back(x)
    assert not library.calls
