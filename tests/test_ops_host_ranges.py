"""Numbers past the C fields that hold them (no GPU needed: nothing is launched)."""
import pytest

from paper_2607_19058_gb300 import _build
from paper_2607_19058_gb300 import skewadam as S


@pytest.fixture(scope="module", autouse=True)
def lib():
    _build.build()
    return S.load()


@pytest.mark.parametrize("name", ["experts", "top_k", "groups", "top_groups", "group_top"])
@pytest.mark.parametrize("past", [1 << 32, -(1 << 32), 1 << 63])
def test_router_refuses_numbers_past_32_bits(name, past):
    kw = dict(experts=8, top_k=2, groups=2, top_groups=1, group_top=1)
    S.Router(**kw)
    kw[name] += past
    with pytest.raises(ValueError, match="32 bits"):
        S.Router(**kw)


@pytest.mark.parametrize("name,what", [("rows", "rows"), ("width", "width")])
def test_embedding_refuses_numbers_past_its_limits(name, what):
    for past in (1 << 32, -(1 << 32), 1 << 62):
        kw = dict(rows=100, width=16)
        kw[name] += past
        with pytest.raises(S.SkewError, match=what):
            S.Embedding(**kw)
    with pytest.raises(S.SkewError, match="scale"):
        S.Embedding(100, 16, scale=1e39)  # infinite in fp32
