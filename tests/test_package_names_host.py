"""The package's names are the binding's, whatever those are at the time."""
import pytest

import paper_2406_18485_amd as P


@pytest.mark.parametrize("name", ["version", "attn_step_fwd", "paged_attn", "make_desc"])
def test_replaced_functions_are_reached(name, monkeypatch):
    first = getattr(P, name)
    assert first is getattr(P.binding, name)
    other = lambda *a, **k: None
    monkeypatch.setattr(P.binding, name, other)
    assert getattr(P, name) is other
    monkeypatch.undo()
    assert getattr(P, name) is first


def test_deleted_functions_are_gone_and_what_the_package_was_given_stays(monkeypatch):
    first = P.binding.version
    assert P.version is first
    monkeypatch.delattr(P.binding, "version")
    with pytest.raises(AttributeError):
        P.version
    monkeypatch.undo()
    mine = lambda: -1
    monkeypatch.setattr(P, "version", mine)
    monkeypatch.setattr(P.binding, "version", lambda: -2)
    assert P.version is mine


def test_names_that_are_not_there():
    with pytest.raises(AttributeError, match="has no attribute 'nothing'"):
        P.nothing
