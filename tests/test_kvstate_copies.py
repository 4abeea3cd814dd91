"""A KVState that has been used in a call is copied, pickled and saved as one that has not, and
lies on one device."""
import copy
import dataclasses
import io
import pickle

import pytest
import torch

from paper_2605_22106_amd import _lib as L


@pytest.fixture
def used(monkeypatch):
    monkeypatch.setattr(L, "_dev", lambda t, name: None if t is None else t.data_ptr())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)     # CPU tensors here
    z = lambda n: torch.arange(n, dtype=torch.int32)  # noqa: E731
    kv = L.KVState(z(4), z(4), z(5), z(5), z(4), z(9), torch.zeros(1, 9, 2, 16, 64),
                   torch.zeros(1, 9, 2, 16, 64), z(9), z(9), z(1), 1, 2, 4, 64, 16, L.F32, 100)
    L._descriptors(kv)
    return kv


def saved(kv):
    f = io.BytesIO()
    torch.save(kv, f)
    f.seek(0)
    return torch.load(f, weights_only=False)          # (of this test's own making)


@pytest.mark.parametrize("make", [copy.deepcopy, copy.copy, lambda kv: pickle.loads(pickle.dumps(kv)),
                                  saved, dataclasses.replace])
def test_copies_of_a_used_state(used, make):
    new = make(used)
    for f in dataclasses.fields(used):
        a, b = getattr(used, f.name), getattr(new, f.name)
        assert torch.equal(a, b) if torch.is_tensor(a) else a == b
    g, t = L._descriptors(new)[1:3]
    assert t._obj.parent == new.parent.data_ptr() and g._obj.num_pages == 9
    assert L._descriptors(used)[2]._obj.parent == used.parent.data_ptr()


def test_a_state_on_two_devices_is_refused(used):
    class Elsewhere(torch.Tensor):
        def get_device(self):
            return 1
    for name in ("parent", "page_table", "v", "free_top"):
        here = getattr(used, name)
        setattr(used, name, here.as_subclass(Elsewhere))
        with pytest.raises(ValueError, match="one device"):
            L._descriptors(used)
        setattr(used, name, here)
    L._descriptors(used)
