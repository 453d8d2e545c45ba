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
SEGMENTS = ((7,), (2, 1, 4), (1, 1, 1, 1, 3))  # tiles of a CTA's segments
SOFT = 2  # softmax warps: one ahead, one behind


class OutOfStep(Exception):
    pass


def explore(stages, per_tile, handovers, segments):
    """Every order of a ring of `stages` stages, `per_tile` to a tile; weights are handed over, and values' products end, by
    `handovers` barriers in turn, one for each place of the ring where there are enough of them."""
    tiles, turn = sum(segments), min(handovers, -(-stages // per_tile))
    total = tiles * per_tile
    begins = {sum(segments[:k]): k for k in range(len(segments))}  # first tile: segment

    # what a softmax warp goes through, and what the values' products arrive on, one after another
    soft, values = [], []
    for k, n in enumerate(segments):
        soft.append(("queries", k))
        for t in range(sum(segments[:k]), sum(segments[:k + 1])):
            soft += [("scores", t), ("rescaled", t), ("weights", t)]
            values += ["stage"] * per_tile + ["tile"]
        soft.append(("segment", k))
        values.append("segment")

    def count(things, upto, what):
        return sum(1 for x in things[:upto] if (x if isinstance(x, str) else x[0]) == what)

    handed = [(count(soft, i, "queries"), count(soft, i, "weights")) for i in range(len(soft) + 1)]
    ended = [tuple(count(values, i, what) for what in ("stage", "tile", "segment")) for i in range(len(values) + 1)]

    def phase(done, k, what):
        """Whether a wait for phase k of a barrier that has completed `done` passes."""
        if done not in (k, k + 1):
            raise OutOfStep(what)
        return done == k + 1

    def like(done, t, turn):  # of `done` tiles in a row, those with t's barrier
        return (done + turn - 1 - t % turn) // turn

    def steps(state):
        loaded, asked, scored, valued, arrived = state[:5]  # loads; scores queued, done; values' tiles queued, arrivals
        warps = state[5:]
        emptied, summed, left = ended[arrived]
        queries, weighted = (min(handed[w][x] for w in warps) for x in (0, 1))  # (a phase of these counts all warps)
        if loaded < total:
            before, slot = loaded // stages, sum(1 for g in range(loaded % stages, emptied, stages))
            if before == 0 or phase(slot, before - 1, "empty"):
                yield (loaded + 1,) + state[1:]
        if asked < tiles and (asked not in begins or phase(queries, begins[asked], "q_full")):
            if asked < 2 or phase(like(weighted, asked - 2, turn), (asked - 2) // turn, "p_full, scores"):
                if loaded >= (asked + 1) * per_tile:
                    yield (loaded, asked + 1) + state[2:]
        if scored < asked:
            yield (loaded, asked, scored + 1) + state[3:]
        if valued < tiles and phase(like(weighted, valued, turn), valued // turn, "p_full, values"):
            yield (loaded, asked, scored, valued + 1) + state[4:]
        # (a segment's end is queued right behind its last tile)
        if arrived < valued * (per_tile + 1) + sum(1 for t, k in begins.items() if t + segments[k] <= valued):
            yield (loaded, asked, scored, valued, arrived + 1) + state[5:]
        for w, at in enumerate(warps):
            if at == len(soft):
                continue
            what, t = soft[at]
            on = (state[:5 + w] + (at + 1,) + state[6 + w:],)
            if what == "scores":
                yield from on if phase(like(scored, t, 2), t // 2, "s_full") else ()
            elif what == "rescaled":  # or not
                yield from on
                if t not in begins:
                    phase(like(summed, t - 1, turn), (t - 1) // turn, "o_done")
            elif what == "segment":
                yield from on if phase(left, t, "segment_done") else ()
            else:
                yield from on

    end = (total, tiles, tiles, tiles, len(values)) + (len(soft),) * SOFT
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


@pytest.mark.parametrize("segments", SEGMENTS, ids=str)
def test_no_order_of_the_warps_brings_a_barrier_out_of_step(ring, segments):
    max_stages, max_tiles, handovers = ring
    for per_tile in (1, 2):
        for stages in range(2 * per_tile, min(max_stages, max_tiles * per_tile) + 1):
            assert explore(stages, per_tile, handovers, segments) > 500


@pytest.mark.parametrize("segments", SEGMENTS, ids=str)
@pytest.mark.parametrize("stages,per_tile", [(3, 1), (6, 2)])
def test_two_barriers_do_not_do_for_three_tiles(stages, per_tile, segments):
    """What the test above finds where tiles that are three apart have barriers of the other parity."""
    with pytest.raises(OutOfStep, match="p_full, values"):
        explore(stages, per_tile, 2, segments)
