"""The two pieces of shared memory through which an epilogue warp of the many-row product hands its outputs to the copy
engine, as a model on the CPU: a piece is written again only when every store of it has been read.  The rule by which a
chunk waits is taken from the kernel's source; the copy engine is as slow as it may be."""
import re
from pathlib import Path

import pytest

SRC = (Path(__file__).resolve().parents[1] / "paper_2502_06282_b200" / "csrc" / "jk_linear_pair.cu").read_text()


def wait_rule():
    """The condition under which all stores but the latest have to have been read (otherwise: all), as Python."""
    text = re.search(r"if \((wide_out && \(OUT8 [^;]*)\) lp_put_read<1>\(\);\s*else lp_put_read<0>\(\);", SRC).group(1)
    for a, b in (("a.out_type == JK_ROWS_T", "is_t"), ("&&", " and "), ("||", " or "), ("!", " not ")):
        text = text.replace(a, b)
    return text


def run(tiles, n_out, n_tile, epi, gated, share, out8):
    """tiles: the weight tiles of a pair, in its order; one warp of the quarter's `share`."""
    chunks = 32 // epi // (1 + gated)
    rule, pending = wait_rule(), []                      # pieces of the stores that may still be read, oldest first
    for wt in tiles:
        first = True
        for c in range(chunks):
            q = share * chunks + c if share < epi // 8 else (share + 1) * chunks - 1 - c
            if wt * n_tile + q * 32 >= n_out:            # no output: nothing is waited for, written or stored
                continue
            left = 1 if eval(rule, dict(wide_out=True, OUT8=out8, is_t=not out8, first=first)) else 0
            pending = pending[len(pending) - left:] if left else []
            first = False
            assert c & 1 not in pending, "a piece is written while a store of it may be reading"
            pending.append(c & 1)


@pytest.mark.parametrize("out8", [False, True])
@pytest.mark.parametrize("gated", [False, True])
def test_pieces_are_written_when_their_stores_have_been_read(gated, out8):
    n_tile = 128 if gated else 256
    for live in range(32, n_tile + 1, 32):               # outputs of the last weight tile
        n_out = 2 * n_tile + live
        for tiles in ([2, 0], [0, 2], [2, 2], [0, 1, 2], [2, 1, 2, 0], [2, 2, 2]):
            for share in range(2):
                run(tiles, n_out, n_tile, 8, gated, share, out8)


def test_lanes_meet_before_an_aligned_cluster_barrier():
    """The last outputs of a shared f32 tile leave lanes at different places; the barrier wants the warp together."""
    text = (Path(__file__).resolve().parents[1] / "paper_2502_06282_b200" / "csrc" / "jk_linear.cu").read_text()
    before = [re.sub(r"//[^\n]*", "", part).rstrip() for part in re.split(r'asm volatile\("barrier\.cluster\.arrive', text)[:-1]]
    assert len(before) == 2
    assert before[1].endswith("__syncwarp();")
