"""CPU tests of the attention binding: operands other than the record's are refused before the library is called."""
import pytest
import torch

A = pytest.importorskip("paper_2504_13850_amd.api")


def test_attention_refuses_operands_of_another_record():
    t = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    i = torch.zeros(1, dtype=torch.int32)
    ok = dict(q=t(4, 2, 8), k=t(6, 1, 8), v=t(6, 1, 8), out=t(4, 2, 8))
    a = A.make_attn(**ok, q_begin=i, q_end=i, k_begin=i, k_end=i, max_q=4, max_k=4)
    lse = t(2, 4, dt=torch.float32)
    for bad in (dict(q=t(3, 2, 8)), dict(k=t(5, 1, 8)), dict(v=t(6, 1, 4)), dict(out=t(4, 2, 8, dt=torch.float32)), dict(q=t(4, 2, 16)[..., :8]),
                dict(lse=t(2, 3, dt=torch.float32)), dict(lse=t(2, 4)), dict(lse=t(2, 8, dt=torch.float32)[:, ::2])):
        x = {**ok, "lse": lse, **bad}
        with pytest.raises(A.FoError):
            A.fo_attn_fwd(a, x["q"], x["k"], x["v"], x["out"], x["lse"])
        with pytest.raises(A.FoError):
            A.fo_attn_bwd(a, x["q"], x["k"], x["v"], x["out"], x["lse"], ok["out"], ok["q"], ok["k"], ok["v"])
