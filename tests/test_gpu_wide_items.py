"""Wide attention items of every short length: with one to six tiles, and whole or open last tiles.

Before each checked call another one fills the rings in LDS with values near 2^100, so that a tile
read before its copy is there cannot look like the right one."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from paper_2608_00814_amd import ooo
from test_gpu_short_parts import check

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from batch_harness import Batch
    from cache8_harness import Batch8


def shared_items(b, plan):
    """Tiles of the plan's wide items over the prompt, from the records (csrc/paged_plan.h)."""
    raw = plan.cpu().numpy()
    ints = lambda at, n: raw[at:at + 4 * n].view(np.int32)  # noqa: E731
    n = int(ints(40, 1)[0])  # the head: key[8], rows, shared_block, shared_items
    up = lambda x: (x + 63) // 64 * 64  # noqa: E731
    seqs, q = len(b.rows), b.n_rows * (b.Hq // b.Hkv)
    workers = max(torch.cuda.get_device_properties(0).multi_processor_count // b.Hkv, 1)
    shared = (q + 127) // 128 if b.shared else 0
    blocks = shared + seqs + q // 128 + seqs + q // 32 + (q // 32 + 1 if b.shared else 0)
    at = up(64 + 16 * blocks)            # behind the head and the blocks' slots
    at = up(at + 4 * (seqs + 1))         # the sequences' first blocks
    at = up(at + 4 * (workers + 1))      # the first items of workers,
    at = up(at + 4 * (8 * workers + 1))  # and of waves
    items = raw[at:at + 64 * n].view(np.int32).reshape(n, 16)
    assert (items[:, 0] == 1).all() and (items[:, 7] == b.shared).all()
    return (items[:, 6] - items[:, 5]).tolist()


# With 64 KV heads a head has four workers: three for the prompt, a third of its tiles each.  With one it has one
# worker a tile.
@pytest.mark.parametrize("tiles,Hkv,shared", [(1, 1, 64 * 6), (2, 64, 64 * 6), (3, 64, 64 * 9), (4, 64, 64 * 12),
                                              (5, 64, 64 * 15), (6, 64, 64 * 18), (1, 1, 64 * 6 - 5),
                                              (2, 64, 64 * 6 - 1), (3, 64, 64 * 9 - 33), (4, 64, 64 * 12 - 63),
                                              (6, 64, 64 * 18 - 7)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("eight", [False, True])
def test_items_of_few_tiles(eight, D, tiles, Hkv, shared):
    kind, plan = (Batch8, ooo.paged_plan8) if eight else (Batch, ooo.paged_plan)
    more = {"quick": True} if eight else {}

    def make(seed):
        return kind("bf16", Hkv, Hkv, D, 32, [30, 40, 20], [3, 0, 9], shared=shared, seed=seed, **more)
    b = make(1)
    assert shared_items(b, plan(b.batch)) == [tiles] * (3 if Hkv > 1 else 6)
    check(make, 3)
