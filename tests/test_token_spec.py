"""Sizes of the model over tokens that are refused before a parameter is laid out (no GPU)."""
import pytest

from paper_2509_26092_gb300.token_step import TokenSpec


@pytest.mark.parametrize("kw", [dict(hidden=-8), dict(hidden=-64), dict(hidden=12), dict(chosen=0), dict(chosen=5),
                                dict(chosen=-1), dict(experts=-1), dict(experts=-4, chosen=-5), dict(experts=1025)], ids=str)
def test_layers_of_experts_that_are_none(kw):
    with pytest.raises(ValueError):
        TokenSpec(64, 1, 10, **{"experts": 4, "hidden": 16, **kw})


def test_every_parameter_has_a_place_of_its_own():
    for hidden in (0, 8, 200):
        spec = TokenSpec(64, 2, 10, 4, hidden)
        ends = [(e.offset, e.offset + e.numel) for e in spec.entries]
        assert all(a < b for a, b in ends) and all(b <= c for (_, b), (c, _) in zip(ends, ends[1:])) and ends[-1][1] <= spec.n_flat
        assert spec.by_name["layer1.up.w"].shape == (4, hidden or 256, 64)
