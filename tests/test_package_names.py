"""The package shows its binding's names as they are now, not as they were when first looked up."""
import pytest

import paper_2507_16768_b200 as wg


@pytest.mark.parametrize("name", ["wg_beam_select", "wg_decode_step", "WG_BEAM_NORM_FULL"])
def test_a_replaced_name_is_seen(monkeypatch, name):
    before = getattr(wg, name)
    assert before is getattr(wg.binding, name)
    other = object()
    monkeypatch.setattr(wg.binding, name, other)
    assert getattr(wg, name) is other
    monkeypatch.undo()
    assert getattr(wg, name) is before


def test_an_unknown_name_is_refused():
    with pytest.raises(AttributeError, match="no attribute 'wg_nothing'"):
        wg.wg_nothing


def test_a_name_of_the_package_itself_goes_first(monkeypatch):
    before = wg.wg_beam_select
    monkeypatch.setattr(wg, "wg_beam_select", 5)
    assert wg.wg_beam_select == 5 and wg.binding.wg_beam_select is before
    monkeypatch.undo()
    assert wg.wg_beam_select is before


def test_a_name_that_is_gone_is_refused(monkeypatch):
    assert wg.WG_BEAM_NORM_NONE == 2
    monkeypatch.delattr(wg.binding, "WG_BEAM_NORM_NONE")
    with pytest.raises(AttributeError, match="no attribute 'WG_BEAM_NORM_NONE'"):
        wg.WG_BEAM_NORM_NONE
