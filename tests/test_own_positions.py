"""CPU: which caches are noted to hold tokens at rotary positions other than their slots, and that Decoder.step asks for positions behind them
before it touches anything."""
from types import SimpleNamespace

import numpy as np
import pytest

from paper_2509_24381_amd.binding import CacheSet, RsError, _note_positions, _positions_arg, int_array
from paper_2509_24381_amd.decode import Decoder


def cache(length, own=False):
    kv = SimpleNamespace(own_positions=own, asked=0)

    def held(layer):
        kv.asked += 1
        return length

    kv.length = held
    return kv


def test_three_axes_that_are_the_slots_or_not():
    """Requests of 3, 0 and 2 new tokens behind 5, 9 and 0 older ones; one number of one axis is enough."""
    slots = np.concatenate([np.arange(5, 8), np.arange(0, 2)])
    positions = np.repeat(slots, 3).reshape(5, 3)
    kvs = [cache(8), cache(9), cache(2)]
    _note_positions(kvs, int_array([3, 0, 2]), _positions_arg(positions), 0)
    assert [kv.own_positions for kv in kvs] == [False] * 3 and kvs[1].asked == 0
    for row, axis, which in ((0, 0, 0), (2, 2, 0), (3, 1, 2), (4, 0, 2)):
        other = positions.copy()
        other[row, axis] += 1
        kvs = [cache(8), cache(9), cache(2)]
        _note_positions(kvs, int_array([3, 0, 2]), _positions_arg(other), 0)
        assert [kv.own_positions for kv in kvs] == [i == which for i in range(3)]
    kvs = [cache(8, own=True), cache(9), cache(2)]   # once noted, it stays
    _note_positions(kvs, int_array([3, 0, 2]), _positions_arg(positions), 0)
    assert kvs[0].own_positions and not kvs[2].own_positions


def test_one_axis():
    kvs = [cache(4), cache(1)]
    _note_positions(kvs, int_array([2, 1]), int_array([2, 3, 7]), 0, axes=1)
    assert [kv.own_positions for kv in kvs] == [False, True]


def test_a_step_asks_for_positions():
    kvs = CacheSet.__new__(CacheSet)
    kvs.caches, kvs.n = [cache(8), cache(9, own=True)], 2
    dec = Decoder.__new__(Decoder)
    dec.ctx, dec.blocks, dec.layers = SimpleNamespace(cfg=None), (0, 1, 2), []
    with pytest.raises(RsError, match=r"kvs\[1\].*positions"):
        dec.step(kvs, [1, 1], None)
