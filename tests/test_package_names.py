"""The package's names are the binding's, at every access."""
import pytest

import paper_2403_11805_amd as kvs
from paper_2403_11805_amd import binding


@pytest.mark.parametrize("name", ["kv_record_bytes", "kv_attend_tokens", "Shape"])
def test_what_is_replaced_in_the_binding_is_replaced_in_the_package(monkeypatch, name):
    before = getattr(kvs, name)
    assert before is getattr(binding, name)
    other = object()
    monkeypatch.setattr(binding, name, other)
    assert getattr(kvs, name) is other
    monkeypatch.undo()
    assert getattr(kvs, name) is before


def test_unknown_names():
    with pytest.raises(AttributeError, match="kv_nothing"):
        kvs.kv_nothing
    assert kvs.binding is binding
