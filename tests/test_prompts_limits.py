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


@pytest.mark.parametrize("change,code", [
    ({"keep_len": FAKE + 64, "len_out": FAKE + 64}, -2),                                     # the kernel reads it as one that nothing writes
    ({"keep_len": FAKE + 64, "len_out": FAKE + 68}, -2), ({"keep_len": FAKE + 68, "len_out": FAKE + 64}, -2),
    ({"len_out": FAKE + 4}, -2), ({"len_out": FAKE - 4}, -2),
    ({"keep_len": FAKE + 64, "len_out": FAKE + 66}, -7)])
def test_new_lengths_overlap_neither_the_lengths_nor_what_to_keep(lib, change, code):
    """(Two sequences: eight bytes each.)"""
    assert lib.mcsd_evict_rows(_evict(len=FAKE, **change), _cache()) == code


def test_arrays_side_by_side_are_no_overlap(lib):
    """(Taken as far as the descriptor's last check: more layers than a grid counts.)"""
    for change in ({"keep_len": FAKE + 64, "len_out": FAKE + 72}, {"keep_len": FAKE + 64, "len_out": FAKE + 56}, {"len_out": FAKE + 8}, {"len_out": FAKE - 8},
                   {"keep_len": FAKE, "len_out": None}):
        assert lib.mcsd_evict_rows(_evict(n_layers=1 << 40, **change), _cache()) == -10


@pytest.mark.parametrize("temperature,code", [(1.2e-38, -1), (4.3e-39, -1), (4.2e-39, -5), (3.0e-39, -5), (2.9e-39, -5)])
def test_temperatures_whose_factor_is_out_of_range(lib, temperature, code):
    """log2(e) / temperature has to be a float32: up to 2^128 / 1.4427 = 1 / 4.2397e-39. (Null logits end the calls that pass.)"""
    assert lib.mcsd_token_logprobs(_logprobs(temperature=temperature, logits=None)) == code
