"""CPU tests of what the binding of the sampling operators keeps and refuses by itself."""
import contextlib

import pytest
import torch

from paper_2602_24082_amd import binding as pp

NAMES = ("page_table", "seq_len", "held", "refs")


def _cache(monkeypatch):
    monkeypatch.setattr(pp, "_on_gpu", lambda t: None)
    return pp.make_cache(3, 4, 9, 16, "cpu")


@pytest.mark.parametrize("name", NAMES)
def test_a_cache_keeps_the_memory_that_calls_go_to(monkeypatch, name):
    """Another tensor in an attribute's place would free what the descriptor points to."""
    c = _cache(monkeypatch)
    t, at = getattr(c, name), getattr(c._desc, name)
    for other in (t + 1, t.clone(), None):
        with pytest.raises(AttributeError):
            setattr(c, name, other)
    with pytest.raises(AttributeError):
        delattr(c, name)
    assert getattr(c, name) is t and t.data_ptr() == at


def test_a_cache_changes_in_place(monkeypatch):
    c = _cache(monkeypatch)
    c.seq_len += 2
    c.held[1] = 1
    c.refs.copy_(torch.arange(9))
    c.page_table = c.page_table
    assert c.seq_len.tolist() == [2, 2, 2] and c.held.tolist() == [0, 1, 0] and c.refs[8] == 8
    for name in NAMES:
        assert getattr(c, name).data_ptr() == getattr(c._desc, name)


@pytest.mark.parametrize("name,value", [("num_pages", 8), ("page_size", 32), ("index", 1), ("ref", None)])
def test_a_cache_keeps_its_sizes(monkeypatch, name, value):
    """Pools are checked by them, and the kernels go by the descriptor's."""
    c = _cache(monkeypatch)
    with pytest.raises(AttributeError):
        setattr(c, name, value)


def test_a_cache_takes_a_callers_own_attributes(monkeypatch):
    c = _cache(monkeypatch)
    c.step = 1
    c.step = 2
    del c.step
    assert not hasattr(c, "step")


@pytest.mark.parametrize("given,want", [({}, 1), ({"parents": True}, 6), ({"parents": True, "max_children": 2}, 2), ({"max_children": 3}, 3)])
def test_children_of_a_tree_are_all_tried_unless_said_otherwise(monkeypatch, given, want):
    seen = []

    class Library:
        def pp_verify_draft(self, *args):
            seen.append(args)
            return 0

    monkeypatch.setattr(pp, "lib", Library)
    monkeypatch.setattr(pp, "_on_gpu", lambda t: None)
    monkeypatch.setattr(pp, "_raw_stream", lambda dev: None)
    monkeypatch.setattr(pp, "_device_of", lambda dev: contextlib.nullcontext())
    monkeypatch.setattr(pp, "pp_verify_workspace_size", lambda *a: 256)
    z = lambda dtype: torch.zeros(2, 6, dtype=dtype)
    kw = dict(given, parents=z(torch.int32)) if "parents" in given else given
    pp.pp_verify_draft(torch.zeros(2, 6, 10), z(torch.int32), z(torch.float32), **kw)
    assert seen[0][:5] == (2, 6, 10, pp.PP_FP32, want)
