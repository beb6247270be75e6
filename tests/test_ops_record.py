"""CPU tests of the attention's record: numbers outside their fields."""
import pytest
import torch

A = pytest.importorskip("paper_2504_13850_amd.api")
I = torch.zeros(1, dtype=torch.int32)
T = torch.zeros((4, 2, 8), dtype=torch.bfloat16)


def _make(max_q=4, max_k=4, **kw):
    return A.make_attn(T, T, T, T, I, I, I, I, max_q, max_k, **kw)


@pytest.mark.parametrize("kw", [dict(max_q=1 << 40), dict(max_k=1 << 31), dict(max_q=-(1 << 40)), dict(mask=1 << 40),
                                dict(scale=1e300), dict(cap=1e39), dict(p=-1e60), dict(max_q=4.5)],
                         ids=lambda k: ",".join(f"{n}={v}" for n, v in k.items()))
def test_refused(kw):
    """By the record's maker, or, as an infinity in 32 bits, by the library's checks."""
    with pytest.raises(A.FoError):
        A.fo_attn_workspace(_make(**kw))


@pytest.mark.parametrize("seed,offset", [(-1, 0), (1 << 64, 1 << 32), (-(1 << 63), -1), ((1 << 64) + 5, (1 << 32) + 7)])
def test_seed_and_offset_count_modulo_their_words(seed, offset):
    """As the dropout calls take them: a layer draws the same numbers through both."""
    a = _make(seed=seed, offset=offset)
    assert (a.seed, a.offset) == (seed % (1 << 64), offset % (1 << 32))
