"""Whether a piece overwrites keys that it sees, against a simulation of the slots it is written to."""
import random

import pytest
import torch

from paper_2602_11937_b200 import paging

BLOCK = 16


def simulated(table, window, blocks, length, new):
    """The keys that the last `new` tokens see, in the slots that hold them after the append: is one of them another's?"""
    if new <= 0 or length <= 0 or length > len(table) * BLOCK:
        return False
    holder = {}
    seen = range(max(0, length - new + 1 - window), length)
    for p in seen:
        if 0 <= table[p // BLOCK] < blocks:
            holder[(table[p // BLOCK], p % BLOCK)] = p
    return any(0 <= table[p // BLOCK] < blocks and holder[(table[p // BLOCK], p % BLOCK)] != p for p in seen)


@pytest.mark.parametrize("window, ring", [(1, 2), (16, 2), (17, 3), (40, 4), (128, 9), (128, 12), (100, 8)])
def test_rings(window, ring):
    width = 40
    table = (torch.arange(width) % ring).int()[None]
    most = 16 * ring + 1 - window
    for length in (most + window, 400, 401, 415, 639, 640):
        for new in sorted({0, 1, 2, most - 1, most, most + 1, most + 9, 16 * ring, 16 * ring + 1, min(length, 300)}):
            if 0 <= new <= length:
                got = paging.window_keys_lost([table], [window], [ring], torch.tensor([length], dtype=torch.int32),
                                              torch.tensor([new]), new)
                assert got.item() == simulated(table[0].tolist(), window, ring, length, new), (length, new)
                if length - new >= window:          # the window before the piece is all there
                    assert got.item() == (new > most)


def test_random_tables_of_several_layers():
    r = random.Random(3)
    for _ in range(300):
        batch, width, layers = r.randint(1, 4), r.randint(1, 20), r.randint(1, 3)
        blocks = [r.choice((2, 5, 30, 200)) for _ in range(layers)]
        windows = [r.choice((1, 9, 33, 128, 2 ** 31 - 1)) for _ in range(layers)]
        tables = []
        for n in blocks:
            t = torch.tensor([[r.choice((-1, n, *range(n))) if r.random() < .3 else (7 * b + j) % n for j in range(width)]
                              for b in range(batch)], dtype=torch.int32)
            tables.append(t)
        lens = [r.choice((0, -3, width * BLOCK + 1, r.randint(1, width * BLOCK))) for _ in range(batch)]
        new = [r.choice((0, 1, r.randint(0, max(n, 0)), r.randint(0, 60))) for n in lens]
        got = paging.window_keys_lost(tables, windows, blocks, torch.tensor(lens, dtype=torch.int32), torch.tensor(new), sum(new))
        assert got.shape == (layers, batch)
        for i in range(layers):
            for b in range(batch):
                assert got[i, b].item() == simulated(tables[i][b].tolist(), windows[i], blocks[i], lens[b], new[b])


def test_blocks_twice():
    t = torch.tensor([[0, 1, 2, 3], [4, 5, 4, 6], [7, -1, -1, 8]], dtype=torch.int32)
    assert paging.blocks_twice([t, t + 9]).tolist() == [[False, True, False], [False, True, True]]
    assert not paging.blocks_twice([paging.linear_block_table(3, 50)]).any()
    assert paging.blocks_twice([paging.ring_block_table(3, 40, 5)]).all() and not paging.blocks_twice([paging.ring_block_table(3, 40, 4)]).any()
