"""The package's names are the binding's, now and after one of them was replaced there."""
import importlib

import pytest

import paper_2502_00299_b200 as ck
from paper_2502_00299_b200 import binding


@pytest.mark.parametrize("name", ["attend_paged", "compress_layer", "lib", "ChunkKVError"])
def test_a_name_replaced_in_the_binding_is_seen_through_the_package(monkeypatch, name):
    was = getattr(ck, name)
    assert was is getattr(binding, name) and getattr(ck, name) is was
    new = object()
    monkeypatch.setattr(binding, name, new)
    assert getattr(ck, name) is new
    monkeypatch.undo()
    assert getattr(ck, name) is was


def test_every_name_is_there():
    assert sorted(ck.__all__) == sorted(set(ck.__all__))
    for name in ck.__all__:
        assert getattr(ck, name) is getattr(binding, name), name
    with pytest.raises(AttributeError):
        ck.no_such_call
    with pytest.raises(ImportError):
        importlib.import_module("paper_2502_00299_b200.no_such_module")
