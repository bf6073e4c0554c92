"""Parts of a few tiles in the wide attention kernels: what an item reads has landed.

Before each checked call another one fills the rings in LDS with values near 2^100, so that a tile
read before its copy is there cannot look like the right one."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from batch_harness import Batch
from cache8_harness import Batch8

pytestmark = pytest.mark.gpu


def waits(tiles, plain, wave, rule):
    """Copies that a barrier promises and the waits of a wave's loop do not: a wave asks for K and V of
    `tiles` tiles and goes over them, up to tile `plain` with a body that always waits until two copies
    are on their way.  rule: such a run begins only where K of tile n + 4 exists."""
    asked, missing = [], []

    def ask(kind, n):
        if n < tiles:
            asked.append((kind, n))

    def barrier(m, left):
        here = asked[:max(len(asked) - left, 0)]
        missing.extend(x for x in (("K", m), ("V", m - 1)) if 0 <= x[1] < tiles and x not in here)

    def careful(m):
        barrier(m, 2 if m + 2 < tiles else 1 if m < tiles else 0)

    for kind, n in (("K", 0), ("K", 1), ("V", 0), ("K", 2)):
        ask(kind, n)
    careful(0)
    ask("V", 1)
    ask("K", 3)
    careful(1)
    if wave:
        ask("V", 2)
    ask("K", 4)
    n, in_run = 0, False
    while n < tiles:
        in_run = n < plain and (in_run or not rule or n + 4 < tiles)
        for first in ((True, False) if wave else (False, True)):  # wave B's barrier comes first
            if first:
                barrier(n + 2, 2) if in_run else careful(n + 2)
            elif in_run:
                asked.append(("V", n + 2 + wave))
            else:
                ask("V", n + 2 + wave)
        if in_run:
            asked.append(("K", n + 5))
        else:
            ask("K", n + 5)
        n += 1
    return missing


def check(make, quiet):
    loud = make(seed=9)
    loud.v.copy_(torch.full_like(loud.v, 0x7E) if loud.v.dtype == torch.uint8 else torch.full_like(loud.v, 2.0 ** 100))
    if hasattr(loud, "vs"):
        loud.vs.fill_(127 + 91)  # 448 times 2^91
    b = make(seed=quiet)
    out, ws = torch.full_like(b.q, 7.0), None
    loud.attend()
    b.check(b.attend(out, ws))


SHAPES = [([70, 1], [100, 20], 600), ([150, 64, 3], [261, 300, 700], 1000), ([200], [0], 0), ([300], [150], 0),
          ([1] * 70, [5] * 70, 2048), ([64, 64], [130, 190], 0)]


@pytest.mark.parametrize("rows,lens,shared", SHAPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("eight", [False, True])
def test_short_parts(eight, D, rows, lens, shared):
    kind = Batch8 if eight else Batch
    check(lambda seed: kind("bf16", 8, 2, D, 64, rows, lens, shared=shared, pad=1, seed=seed), 3)
