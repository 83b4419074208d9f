"""Limits of the operators of prompts and long conversations, checked on the host before anything is enqueued (fake pointers are never used)."""
import pytest

from paper_2401_06706_b200 import binding, build
from test_prompts_host import FAKE, _attend, _cache, _chunk, _evict, _logprobs, _weigh


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


@pytest.mark.parametrize("n_tokens,fits", [(1 << 24, False), ((1 << 24) - 2, False), ((1 << 24) - 3, True), (100, True)])
def test_rows_of_a_chunk_are_counted_in_32_bits(lib, n_tokens, fits):
    """128 query heads a key head and chunks of up to 2^24 tokens: rows, and those of a last block beside them, stay below 2^31. (A call that fits is
    refused for its workspace or stops at its null pointers here.)"""
    d = _chunk(n_heads=256, max_new=1 << 24, n_tokens=n_tokens, q_token_stride=256 * 128, out_token_stride=256 * 128, workspace=None)
    assert _attend(lib, d) == (-8 if fits else -10)
    assert _weigh(lib, d, q=None) == (-1 if fits else -10)
    assert (lib.mcsd_chunk_attention_workspace_bytes(d, _cache()) > 0) == fits
