"""Sequences whose last tile of rows has any number of tokens, in groups of every size: rows without a token share their warp with rows
that have one."""
import pytest

from test_gpu_chunk_attn import Case
from test_gpu_prompt_attn import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rest", range(1, 17))
def test_prompts(rest):
    run([rest, 640 + rest, 1200 + rest], seed=rest)                  # groups of 64
    run([96 + rest, 48 + rest], seed=rest, hkv=2)                    # groups of 16


@pytest.mark.parametrize("rest", [1, 2, 3, 5, 6, 7, 13, 15])
@pytest.mark.parametrize("kv", ["fp8", "bf16", "fp4"])
def test_chunks(kv, rest):
    Case(kv, [900, 2100], [640 + rest, 704 + rest], hkv=8, seed=rest).call().verify()
    Case(kv, [1300, 2000], [640 + rest, 400], 100, hkv=8, seed=rest).call().verify()       # groups of 32
    Case(kv, [40, 333], [rest, 16 + rest], seed=rest).call().verify()
