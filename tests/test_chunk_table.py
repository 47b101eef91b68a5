"""DeviceChunkTable as the library's calls see it: the struct they are given always holds the arrays' present addresses, and a
table that was used can be copied and pickled."""
import copy
import pickle

import pytest
import torch

from paper_2601_21109_b200 import binding as cwl

ARRAYS = ("offsets", "rank", "scale", "rung", "flags", "n_chunks")


def used():
    t = cwl.DeviceChunkTable.from_host([0, 3, 8], [4, 8], [1.0, 0.5], [1, 0], device="cpu")
    t.c_struct()
    return t


def points_at(t):
    c = t.c_struct()
    return all(getattr(c, n) == getattr(t, n).data_ptr() for n in ARRAYS) and c.capacity == t.capacity


@pytest.mark.parametrize("name", ARRAYS)
def test_the_struct_follows_arrays_that_move(name):
    t = used()
    assert points_at(t)
    old = getattr(t, name).clone()
    setattr(t, name, old)                                      # another tensor
    assert points_at(t)
    getattr(t, name).set_(torch.zeros(100, dtype=old.dtype))   # other storage
    assert points_at(t)
    getattr(t, name).data = torch.zeros(50, dtype=old.dtype)
    assert points_at(t)
    getattr(t, name).resize_(1 << 16)                          # moves
    assert points_at(t)
    t.capacity = 1
    assert points_at(t)


def test_a_used_table_can_be_copied_and_pickled():
    t = used()
    for u in (copy.deepcopy(t), pickle.loads(pickle.dumps(t))):
        assert points_at(u) and u.capacity == 2
        for n in ARRAYS:
            assert torch.equal(getattr(u, n), getattr(t, n)) and getattr(u, n).data_ptr() != getattr(t, n).data_ptr()
    shallow = copy.copy(t)
    assert points_at(shallow)
    shallow.rank = t.rank.clone()
    assert points_at(shallow) and points_at(t)
