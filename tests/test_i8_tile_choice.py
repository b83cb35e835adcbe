"""Which kernel a product with 8-bit weights takes (csrc/lordba_i8_choice.h, compiled for the host: no GPU), and that the shapes of the GPU tests reach every one
of them in every way of ending a tile and a contraction."""
import os
import subprocess

import pytest

import i8_shapes as shapes
from paper_2605_24058_amd import binding

PROGRAM = r"""
#include <cstdio>
#include "lordba_i8_choice.h"
int main() {
    long long T, cols, n;
    int digits, gated, aligned;
    while (std::scanf("%lld %lld %lld %d %d %d", &T, &cols, &n, &digits, &gated, &aligned) == 6) {
        const Choice c = i8_choice(T, cols, n, digits, gated != 0);
        const TileCost t = (gated ? kGatedTiles : kTiles)[c.tile];
        std::printf("%d %d %u %d %d %lld\n", i8_own_rows(T, cols, digits, gated != 0, aligned != 0), c.tile, c.splits, t.channels, t.tokens,
                    static_cast<long long>(i8_pieces(cols)));
    }
}
"""
SIDE_BY_SIDE = {False: {0: 1, 1: 1, 2: 1, 3: 2, 4: 2, 5: 4, 6: 4}, True: {0: 1, 1: 1, 2: 1, 3: 2, 4: 2, 6: 2}}     # waves on a step's columns, 64 each
SLOTS = 4                                                                                                        # of the ring


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    d = tmp_path_factory.mktemp("choice")
    (d / "choose.cpp").write_text(PROGRAM)
    subprocess.run([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-I", binding._CSRC, str(d / "choose.cpp"), "-o", str(d / "choose")],
                   check=True, capture_output=True, timeout=120)

    def ask(calls):
        """[(own, tile, splits, channels, tokens, pieces)] of [(T, columns, n, digits, gated, aligned)]"""
        text = "".join("%d %d %d %d %d %d\n" % c for c in calls)
        out = subprocess.run([str(d / "choose")], input=text, check=True, capture_output=True, text=True, timeout=60).stdout
        got = [tuple(int(v) for v in line.split()) for line in out.splitlines()]
        assert len(got) == len(calls)
        return got
    return ask


def tile_of(gated, tile):
    return 4 if gated and tile == 5 else tile     # (64 x 32 stands for both)


def test_every_tile_is_reached(choose):
    assert set(shapes.TILES) == {(g, d, t) for g in (False, True) for d in (1, 2) for t in SIDE_BY_SIDE[g] if (d, t) != (2, 6)}
    for (gated, digits, tile), some in shapes.TILES.items():
        ends, steps = set(), set()
        for (T, cols, n), (_, t, splits, channels, tokens, pieces) in zip(some, choose([(*s, digits, gated, 0) for s in some])):
            assert (tile_of(gated, t), splits) == (tile, 1), (gated, digits, tile, T, cols, n, t, splits)
            wide, high = channels // (2 if gated else 1), tokens // digits
            ends |= {"whole"} if T % high == 0 and n % wide == 0 and n % 32 == 0 else set()
            ends |= {"odd" if n % 2 else "even" if n % 8 else "eight"} if T >= high and n >= wide and n % 32 else set()
            ends |= {"ragged"} if T % high and n % wide else set()
            steps.add(-(-pieces // SIDE_BY_SIDE[gated][tile]))
        assert ends == {"whole", "odd", "even", "eight", "ragged"}, (gated, digits, tile, ends)
        # (256 x 256 and 256 x 128 tiles of plain products lose to smaller ones up to four and five steps)
        least = {0: 5, 1: 6}.get(tile, 1) if not gated else 1
        assert set(range(least, SLOTS + 5)) <= steps and max(steps) > 20, (gated, digits, tile, steps)


def test_the_addends_come_through_the_ring_from_its_first_full_turn_on(choose):
    for (digits, tile), some in shapes.AHEAD.items():
        steps = set()
        for (T, cols, n), (_, t, splits, channels, tokens, pieces) in zip(some, choose([(*s, digits, 1, 0) for s in some])):
            assert (t, splits) == (tile, 1) and T % (tokens // digits) == 0 and n % (channels // 2) == 0 and n % 8 == 0 and pieces >= SLOTS
            steps.add(pieces)
        assert set(range(SLOTS, SLOTS + 5)) <= steps, (digits, tile, steps)
    assert set(shapes.AHEAD) == {(d, t) for d in (1, 2) for t in (0, 1, 2)}
    for digits, s in shapes.STREAMED.items():
        (_, t, splits, channels, tokens, pieces), = choose([(*s, digits, 1, 0)])
        assert t == 0 and s[0] * s[2] >= 1 << 25 and s[2] % 32 == 0 and pieces > SLOTS
    assert set(shapes.STREAMED) == {1, 2}


def test_every_way_of_sharing_is_reached(choose):
    assert set(shapes.SHARED) == {(g, d, t) for g in (False, True) for d in (1, 2) for t in SIDE_BY_SIDE[g] if t >= 3 and (d, t) != (2, 6)}
    for (gated, digits, tile), some in shapes.SHARED.items():
        for s, (_, t, splits, *_) in zip(some, choose([(*s, digits, gated, 0) for s in some])):
            assert tile_of(gated, t) == tile and splits >= 2, (gated, digits, tile, s, t, splits)


def test_every_way_of_making_rows_is_reached(choose):
    assert set(shapes.OWN_ROWS) == {(g, w) for g in (False, True) for w in (1, 2)}
    for (gated, way), some in shapes.OWN_ROWS.items():
        for s, (own, *_) in zip(some, choose([(*s, 1, gated, 1) for s in some])):
            assert own == way, (gated, s, own)
        assert all(own != 1 for own, *_ in choose([(*s, 1, gated, 0) for s in some]))     # (x off its 16 bytes)
        assert all(own == 0 for own, *_ in choose([(*s, 2, gated, 1) for s in some]))


def test_the_choice_for_any_sizes(choose):
    # tiles that exist, as few workgroups on a shared contraction as there are counters, never on one that has no room for the sums
    sizes = [1, 2, 5, 16, 33, 64, 100, 256, 257, 512, 700, 2048, 4095, 9000, 13824, 40000, 131071]
    calls = [(T, c, n, d, g, 1) for T in sizes for c in sizes for n in sizes for d in (1, 2) for g in (0, 1)]
    for (T, cols, n, digits, gated, _), (_, t, splits, channels, tokens, pieces) in zip(calls, choose(calls)):
        assert 0 <= t < (7 if digits == 1 else 6) and 1 <= splits <= 16 and pieces == -(-cols // 64)
        if splits > 1:
            tiles = -(-(n * (2 if gated else 1)) // channels) * -(-(T * digits) // tokens)
            assert t >= 3 and tiles * splits <= 256 and cols > 1792 and T * digits <= 512 and channels * tokens <= 64 * 64
