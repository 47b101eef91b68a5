"""Workspaces of the head's loss: one made for a call with gradients does for the loss alone, as the tuning path uses it."""
import random

import pytest

from paper_2601_21109_b200 import binding as cwl


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2601_21109_b200 import build
    build.build()


@pytest.mark.parametrize("T,d,V", [(143123, 245, 298359), (76211, 4, 287384), (262144, 64, 262144), (16384, 4096, 32000), (1, 1, 1)])
def test_gradients_workspace_does_for_the_loss(T, d, V):
    w = cwl.cwl_head_loss_workspace_bytes
    alone = w(T, d, V)
    assert 0 < alone <= min(w(T, d, V, True), w(T, d, V, False, True), w(T, d, V, True, True))


def test_over_the_whole_range():
    w, rng = cwl.cwl_head_loss_workspace_bytes, random.Random(1)
    for _ in range(20000):
        T, d, V = (int(2 ** rng.uniform(0, top)) for top in (18.5, 13, 18.2))
        assert 0 < w(T, d, V) <= min(w(T, d, V, True), w(T, d, V, False, True), w(T, d, V, True, True))
