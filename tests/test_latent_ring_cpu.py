"""The barriers of the latent attention kernel without a GPU: all orders in which its warps and the products they queue can
proceed, for each shape of its ring of tiles.

A wait names a phase by its parity alone, so it is right only while its barrier has completed that phase or the one before it:
two phases further on it would hold, one phase further back it would pass. The model has the waits of the kernel's warps
(k_latent_attn.cu), with products and arrivals completing any time after they are queued, in their order; it says whether some
order brings a barrier out of step with a warp that waits for it, and whether all of them end.
"""

import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TILES = 7  # of a CTA
SOFT = 2  # softmax warps: one ahead, one behind


class OutOfStep(Exception):
    pass


def explore(stages, per_tile, handovers, tiles=TILES):
    """Every order of a ring of `stages` stages, `per_tile` to a tile; weights are handed over, and values' products end, by
    `handovers` barriers in turn, one for each place of the ring where there are enough of them."""
    total, turn = tiles * per_tile, min(handovers, -(-stages // per_tile))

    def phase(done, k, what):
        """Whether a wait for phase k of a barrier that has completed `done` passes."""
        if done not in (k, k + 1):
            raise OutOfStep(what)
        return done == k + 1

    def like(done, t, turn):  # of `done` tiles in a row, those with t's barrier
        return (done + turn - 1 - t % turn) // turn

    def ended(arrived):  # the values' arrivals so far, a tile's stages and then the tile: (stages, tiles)
        whole, rest = divmod(arrived, per_tile + 1)
        return whole * per_tile + rest, whole

    def steps(state):
        loaded, asked, scored, valued, arrived = state[:5]  # loads; scores queued, done; values' tiles queued, arrivals
        soft = state[5:]  # of each warp: 3 * tile + what it has behind it of that (nothing, scores, the last tile's values)
        emptied, summed = ended(arrived)
        weighted = min(s // 3 for s in soft)  # (a phase of p_full counts all warps)
        if loaded < total:
            before = (loaded - loaded % stages) // stages
            slot = sum(1 for g in range(loaded % stages, emptied, stages))
            if before == 0 or phase(slot, before - 1, "empty"):
                yield (loaded + 1,) + state[1:]
        if asked < tiles and (asked < 2 or phase(like(weighted, asked - 2, turn), (asked - 2) // turn, "p_full, scores")):
            if loaded >= (asked + 1) * per_tile:
                yield (loaded, asked + 1) + state[2:]
        if scored < asked:
            yield (loaded, asked, scored + 1) + state[3:]
        if valued < tiles and phase(like(weighted, valued, turn), valued // turn, "p_full, values"):
            yield (loaded, asked, scored, valued + 1) + state[4:]
        if arrived < valued * (per_tile + 1):
            yield (loaded, asked, scored, valued, arrived + 1) + state[5:]
        for w, s in enumerate(soft):
            t, at = divmod(s, 3)
            to = None
            if t == tiles:
                continue
            if at == 0:
                if phase(like(scored, t, 2), t // 2, "s_full"):
                    to = s + 1
            elif at == 1:  # its sums may have to be rescaled, or not
                yield state[:5 + w] + (s + 1,) + state[6 + w:]
                if t and phase(like(summed, t - 1, turn), (t - 1) // turn, "o_done"):
                    to = s + 1
            else:
                to = s + 1
            if to is not None:
                yield state[:5 + w] + (to,) + state[6 + w:]

    end = (total, tiles, tiles, tiles, tiles * (per_tile + 1)) + (3 * tiles,) * SOFT
    start = (0,) * (5 + SOFT)
    seen, todo = {start}, [start]
    while todo:
        state = todo.pop()
        following = list(steps(state))
        assert following or state == end, f"nothing can go on from {state}"
        for s in following:
            if s not in seen:
                seen.add(s)
                todo.append(s)
    assert end in seen
    return len(seen)


@pytest.fixture(scope="module")
def ring(tmp_path_factory):
    """MAX_STAGES, MAX_TILES, HANDOVERS of the kernel."""
    from paper_2609_33887_gb300 import build

    try:
        nvcc = build._nvcc()
    except RuntimeError as e:
        pytest.skip(str(e))
    src = tmp_path_factory.mktemp("ring") / "ring.cu"
    src.write_text("""#include "rotary/latent.h"
#include <cstdio>
int main() { std::printf("%d %d %d\\n", bdrot::MAX_STAGES, bdrot::MAX_TILES, bdrot::HANDOVERS); }
""")
    exe = str(src)[:-3]
    r = subprocess.run([nvcc, "-std=c++17", "-I" + build.CSRC, "-I" + os.path.join(build.CSRC, "cache"),
                        "-I" + build.INCLUDE, "-o", exe, str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return [int(v) for v in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]


def test_no_order_of_the_warps_brings_a_barrier_out_of_step(ring):
    max_stages, max_tiles, handovers = ring
    for per_tile in (1, 2):
        for stages in range(2 * per_tile, min(max_stages, max_tiles * per_tile) + 1):
            assert explore(stages, per_tile, handovers) > 1000


@pytest.mark.parametrize("stages,per_tile", [(3, 1), (6, 2)])
def test_two_barriers_do_not_do_for_three_tiles(stages, per_tile):
    """What the test above finds where tiles that are three apart have barriers of the other parity."""
    with pytest.raises(OutOfStep, match="p_full, values"):
        explore(stages, per_tile, 2)
