"""Pieces behind the prompts on stacks whose window layers keep rings of blocks: the same bits as over full caches as long as a ring holds
the piece and the window before it, a refusal that stores nothing beyond."""
import pytest
import torch

from prompt_helpers import D, gen, make_starts
from test_gpu_prefill import ALL, BLOCKS, HKV, HQ, WINDOWS, Model, parts

pytestmark = pytest.mark.gpu
MOST = 25      # window 40, four blocks: 16 * 4 + 1 - 40; the other window, 17 in three blocks, takes 32


def piece(models, new, g, continued, stream=None):
    at, starts = make_starts(new)
    qkv = [torch.randn(at[-1], HQ + 2 * HKV, D, generator=g, device="cuda").bfloat16() for _ in WINDOWS]
    outs = []
    for m in models:
        m.lens += torch.tensor(new, dtype=torch.int32, device="cuda")
        out = [torch.empty(at[-1], HQ, D, dtype=torch.bfloat16, device="cuda") for _ in WINDOWS]
        m.stack.prefill(*parts(qkv), starts, out, continued=continued, stream=stream)
        torch.cuda.synchronize()
        assert m.stack.status.item() == 0
        outs.append(out)
    return outs


@pytest.mark.parametrize("kv", ALL)
def test_pieces_that_fit(kv):
    g = gen(21)
    models = [Model(kv, [100, 37, 0], rings) for rings in (False, True)]
    for m in models:
        m.lens.zero_()
    piece(models, [100, 37, 0], g, False)
    for new in ([MOST, 1, 3], [1, MOST, 0], [MOST, MOST, MOST], [7, 16, 17], [2, 0, 1]):
        full, ring = piece(models, new, g, True, torch.cuda.Stream() if new[0] == 7 else None)
        for a, b in zip(full, ring):
            assert torch.equal(a, b)


def test_longer_pieces_are_refused():
    g = gen(22)
    full, ring = [Model("fp8", [90, 70], rings) for rings in (False, True)]
    for m in (full, ring):
        m.lens.zero_()
    piece([full, ring], [90, 70], g, False)
    kept = [t.clone() for c in ring.caches for t in c]
    with pytest.raises(ValueError, match="too long for the ring of layer 1 .window 40."):
        piece([ring], [2, MOST + 1], g, True)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(kept, (t for c in ring.caches for t in c)))
    piece([full], [2, MOST + 1], g, True)                         # over a full table any length is right
    ring.lens -= torch.tensor([2, MOST + 1], dtype=torch.int32, device="cuda")
    piece([ring], [2, MOST], g, True)


def test_a_table_that_becomes_a_ring():
    """A table without repeats is not looked at again until it changes."""
    g = gen(23)
    m = Model("fp8", [90, 70], False)
    m.lens.zero_()
    piece([m], [90, 70], g, False)
    piece([m], [MOST + 9, 1], g, True)
    m.tables[1].copy_((m.tables[1] // BLOCKS) * BLOCKS + m.tables[1] % BLOCKS % 4)
    with pytest.raises(ValueError, match="layer 1"):
        piece([m], [MOST + 9, 1], g, True)
