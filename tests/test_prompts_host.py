"""Host-side checks of the operators of prompts and long conversations: refusals come back with the documented codes before
anything is enqueued (fake pointers are never used), and the plain statements they are tested against hold by hand."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import ops_reference as ops
import prompts_reference as ref
from paper_2401_06706_b200 import binding, build

FAKE = 0x10000


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def _cache(**kw):
    c = binding.McsdKvCache()
    c.pages, c.n_pages, c.n_heads, c.head_dim, c.page_size = FAKE, 10, 2, 128, 16
    for k, v in kw.items():
        setattr(c, k, v)
    if "page_stride" not in kw:
        c.page_stride = c.n_heads * 16 * 136
    return c


def _chunk(**kw):
    d = binding.McsdChunkDesc()
    d.batch, d.n_heads, d.dtype, d.max_pages, d.max_new, d.n_tokens, d.ld_table = 2, 4, 1, 8, 30, 40, 8
    d.q_token_stride, d.q_head_stride, d.out_token_stride, d.out_head_stride = 512, 128, 512, 128
    d.scale, d.workspace, d.workspace_bytes = 0.1, FAKE, 1 << 40
    for k, v in kw.items():
        setattr(d, k, v)
    return d


SHARED = [({"batch": -1}, -2), ({"n_heads": 0}, -2), ({"n_heads": 5}, -2), ({"n_heads": 2 * 129}, -10), ({"dtype": 0}, -3), ({"dtype": 9}, -3),
          ({"max_pages": -1}, -2), ({"max_new": -1}, -2), ({"max_new": (1 << 24) + 1}, -10), ({"n_tokens": -1}, -2), ({"n_tokens": 1 << 31}, -10),
          ({"reserved": 1}, -2), ({"ld_table": 7}, -7), ({"q_token_stride": -1}, -7), ({"q_head_stride": -1}, -7), ({"scale": float("nan")}, -2),
          ({"scale": float("inf")}, -2), ({"max_pages": 1 << 27, "ld_table": 1 << 27}, -10)]


def _attend(lib, d, c=None, table=FAKE, start=FAKE, cu=FAKE, q=FAKE, out=FAKE, lse=FAKE):
    return lib.mcsd_chunk_attention(d, c or _cache(), table, start, cu, q, out, lse)


def _weigh(lib, d, c=None, table=FAKE, start=FAKE, cu=FAKE, q=FAKE, lse=FAKE, weights=FAKE, decay=1.0, last=0):
    return lib.mcsd_accumulate_weights(d, c or _cache(), table, start, cu, q, lse, weights, decay, last)


@pytest.mark.parametrize("change,code", SHARED)
def test_chunk_refusals(lib, change, code):
    assert _attend(lib, _chunk(**change)) == code
    assert _weigh(lib, _chunk(**change)) == code
    if "scale" not in change:
        assert lib.mcsd_chunk_attention_workspace_bytes(_chunk(**change), _cache()) == 0


@pytest.mark.parametrize("change,code", [({"out_token_stride": 127}, -7), ({"out_head_stride": 127}, -7), ({"out_token_stride": -512, "n_tokens": 1}, -7),
                                         ({"workspace": None}, -8), ({"workspace": FAKE + 16}, -8), ({"workspace_bytes": 0}, -8)])
def test_attention_refusals(lib, change, code):
    assert _attend(lib, _chunk(**change)) == code


def test_chunk_pointers_and_empty_calls(lib):
    for name in ("table", "start", "cu", "q", "out"):
        assert _attend(lib, _chunk(), **{name: None}) == -1, name
    for name in ("table", "start", "cu", "q", "lse", "weights"):
        assert _weigh(lib, _chunk(), **{name: None}) == -1, name
    for name, off in (("table", 2), ("start", 2), ("cu", 2), ("q", 1), ("out", 1), ("lse", 2)):
        assert _attend(lib, _chunk(), **{name: FAKE + off}) == -7, name
    for name, off in (("table", 2), ("start", 2), ("cu", 2), ("q", 1), ("lse", 2), ("weights", 2)):
        assert _weigh(lib, _chunk(), **{name: FAKE + off}) == -7, name
    for change in ({"batch": 0}, {"n_tokens": 0}, {"max_new": 0}):
        assert _attend(lib, _chunk(**change), None, None, None, None, None, None, None) == 0
        assert _weigh(lib, _chunk(**change), None, None, None, None, None, None, None) == 0
    assert _weigh(lib, _chunk(), last=-1) == -2 and _weigh(lib, _chunk(), decay=float("nan")) == -2 and _weigh(lib, _chunk(), decay=float("inf")) == -2
    assert lib.mcsd_chunk_attention(None, _cache(), *[FAKE] * 6) == -1 and lib.mcsd_chunk_attention(_chunk(), None, *[FAKE] * 6) == -1
    assert lib.mcsd_accumulate_weights(None, _cache(), *[FAKE] * 6, 1.0, 0) == -1 and lib.mcsd_accumulate_weights(_chunk(), None, *[FAKE] * 6, 1.0, 0) == -1
    assert lib.mcsd_chunk_attention_workspace_bytes(None, _cache()) == 0
    n = lib.mcsd_chunk_attention_workspace_bytes(_chunk(), _cache())
    assert n > 0 and n % 256 == 0
    # neither the lengths nor the number of tokens of a call matter
    assert lib.mcsd_chunk_attention_workspace_bytes(_chunk(n_tokens=7), _cache()) == n


@pytest.mark.parametrize("change,code", [({"head_dim": 96}, -10), ({"page_size": 8}, -10), ({"n_heads": 0}, -2), ({"n_pages": -1}, -2), ({"pages": None}, -1),
                                         ({"pages": FAKE + 8}, -7), ({"page_stride": 2 * 16 * 136 + 8}, -7)])
def test_cache_refusals(lib, change, code):
    c = _cache(**change)
    assert _attend(lib, _chunk(), c) == code and _weigh(lib, _chunk(), c) == code and lib.mcsd_evict_rows(_evict(), c) == code


def _evict(**kw):
    d = binding.McsdEvictDesc()
    d.batch, d.max_pages, d.keep, d.n_layers, d.ld_table, d.weight_stride, d.layer_stride = 2, 8, 20, 3, 8, 10 * 2 * 16, 10 * 2 * 16 * 136
    d.page_table = d.len = d.weights = FAKE
    d.len_out = 2 * FAKE
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,code", [
    ({"batch": -1}, -2), ({"max_pages": -1}, -2), ({"keep": -1}, -2), ({"sink": -1}, -2), ({"recent": -1}, -2), ({"n_layers": 0}, -2), ({"reserved": 3}, -2),
    ({"ld_table": 7}, -7), ({"layer_stride": 8}, -7), ({"layer_stride": -16}, -7), ({"layer_stride": 16}, -7), ({"weight_stride": 319}, -7), ({"weight_stride": -1}, -7),
    ({"max_pages": 1 << 27, "ld_table": 1 << 27}, -10), ({"n_layers": 1 << 40}, -10), ({"len": None}, -1), ({"page_table": None}, -1), ({"weights": None}, -1),
    ({"len_out": FAKE}, -2), ({"page_table": FAKE + 2}, -7), ({"len": FAKE + 2}, -7), ({"keep_len": FAKE + 2}, -7), ({"weights": FAKE + 2}, -7),
    ({"len_out": FAKE + 2}, -7), ({"batch": 0}, 0)])
def test_evict_refusals(lib, change, code):
    assert lib.mcsd_evict_rows(_evict(**change), _cache()) == code
    assert lib.mcsd_evict_rows(None, _cache()) == -1 and lib.mcsd_evict_rows(_evict(), None) == -1


def _logprobs(**kw):
    d = binding.McsdLogprobDesc()
    d.vocab, d.dtype, d.n_given, d.n_top, d.n_logits, d.ld, d.n_out, d.temperature = 64, 0, 1, 3, 6, 64, 6, 1.0
    d.logits = d.tokens = d.logprobs = d.entropy = d.top_ids = d.top_logprobs = FAKE
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,code", [
    ({"vocab": 0}, -2), ({"vocab": 65537, "ld": 65537}, -10), ({"dtype": 3}, -3), ({"n_given": -1}, -2), ({"n_top": -1}, -2), ({"n_top": 33}, -10), ({"vocab": 2}, -2),
    ({"n_logits": -1}, -2), ({"n_out": -1}, -2), ({"n_out": 1 << 31}, -10), ({"ld": 63}, -7), ({"reserved": 1}, -2), ({"temperature": 0.0}, -5), ({"temperature": -1.0}, -5),
    ({"temperature": float("nan")}, -5), ({"temperature": float("inf")}, -5), ({"temperature": 1e-40}, -5), ({"logits": None}, -1), ({"tokens": None}, -1),
    ({"path_nodes": FAKE, "row_index": FAKE, "path_len": 3, "nodes_per_tree": 2}, -2), ({"path_nodes": FAKE, "path_len": 0, "nodes_per_tree": 2}, -2),
    ({"path_nodes": FAKE, "path_len": 3, "nodes_per_tree": 0}, -2), ({"path_nodes": FAKE, "path_len": 4, "nodes_per_tree": 2}, -2),
    ({"logits": FAKE + 2}, -7), ({"row_index": FAKE + 2}, -7), ({"tokens": FAKE + 2}, -7), ({"logprobs": FAKE + 2}, -7), ({"entropy": FAKE + 2}, -7),
    ({"top_ids": FAKE + 2}, -7), ({"top_logprobs": FAKE + 2}, -7), ({"path_nodes": FAKE + 2, "path_len": 3, "nodes_per_tree": 2}, -7), ({"n_out": 0}, 0), ({"n_logits": 0}, 0)])
def test_logprob_refusals(lib, change, code):
    assert lib.mcsd_token_logprobs(_logprobs(**change)) == code
    assert lib.mcsd_token_logprobs(None) == -1


def test_constants_match_the_header():
    text = open(os.path.join(build.ROOT, "include", "mcsd.h")).read()
    consts = dict(re.findall(r"#define\s+(MCSD_[A-Z0-9_]+)\s+(\d+)", text))
    assert int(consts["MCSD_MAX_GROUP"]) == binding.MAX_GROUP and int(consts["MCSD_MAX_TOP"]) == binding.MAX_TOP


def test_descriptors_have_the_layout_of_the_header(tmp_path):
    """Sizes and the offset of every field, from the C compiler."""
    import subprocess
    pairs = (("mcsd_chunk_desc", binding.McsdChunkDesc), ("mcsd_evict_desc", binding.McsdEvictDesc), ("mcsd_logprob_desc", binding.McsdLogprobDesc))
    lines = [f'printf("%zu\\n", sizeof({name}));' + "".join(f'printf("%zu\\n", offsetof({name}, {f[0]}));' for f in t._fields_) for name, t in pairs]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "mcsd.h"\nint main(void) {' + "\n".join(lines) + "return 0; }\n")
    subprocess.run(["gcc", "-I", os.path.join(build.ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for _, t in pairs:
        want += [ctypes.sizeof(t)] + [getattr(t, f[0]).offset for f in t._fields_]
    assert got == want


# ---------------------------------------------------------------- the plain statements, by hand
def test_reference_chunk_by_hand():
    """Two cached positions and three new tokens: token i sees 3 + i positions."""
    ps, D = 16, 64
    rng = np.random.default_rng(0)
    k, v = rng.standard_normal((5, 1, D)), rng.standard_normal((5, 1, D))
    pages = ops.append(np.zeros((1, 1, ps * (D + 8)), dtype=np.uint8), k, v, np.arange(5), D, ps)
    q = rng.standard_normal((4, 1, D))
    out, lse, _, _ = ref.chunk_attention(q, pages, np.array([[0]]), [2], [0, 3], 9, D, ps, 0.125, 2.0 ** -10)
    kk, vv = (np.stack([ops.row_values(pages, 0, t, D, ps)[i][0] for t in range(5)]) for i in (0, 1))
    weights = np.zeros((1, 1, ps), dtype=np.float32)
    weights[0, 0, :3] = [1.0, 2.0, 7.0]
    got = np.zeros(5)
    for i in range(3):
        s = 0.125 * kk[:3 + i] @ q[i, 0]
        w = np.exp(s) / np.exp(s).sum()
        assert np.allclose(out[i, 0], w @ vv[:3 + i]) and np.allclose(lse[i, 0], np.log(np.exp(s).sum()))
        got[:3 + i] += w * (i >= 1)
    assert np.isnan(out[3]).all()
    after, _ = ref.accumulate(q, lse, pages, weights, np.array([[0]]), [2], [0, 3], 9, D, ps, 0.125, 0.5, 2)
    assert np.allclose(after[0, 0, :5], got + [0.5, 1.0, 0, 0, 0]) and (after[0, 0, 5:] == 0).all()


def test_reference_evict_by_hand():
    ps, D = 16, 64
    pages = np.arange(ps * (D + 8), dtype=np.int64).astype(np.uint8).reshape(1, 1, 1, -1)
    w = np.zeros((1, 1, 1, ps), dtype=np.float32)
    w[0, 0, 0, :8] = [0, 5, 3, np.nan, 5, 9, 1, 0]
    p, after, n = ref.evict(pages, w, np.array([[0]]), np.array([8]), [5], 1, 1, D, ps)
    assert n.tolist() == [5] and after[0, 0, 0, :5].tolist() == [0, 5, 5, 9, 0]         # rows 0, 1, 4, 5, 7
    assert np.isnan(after[0, 0, 0, 3]) == False and after[0, 0, 0, 5:8].tolist() == [9, 1, 0]
    for dst, src in enumerate([0, 1, 4, 5, 7]):
        assert (p[0, 0, 0, dst * 32:(dst + 1) * 32] == pages[0, 0, 0, src * 32:(src + 1) * 32]).all()


def test_reference_logprobs_by_hand():
    row = np.array([0.0, np.log(2.0), np.log(2.0), -np.inf])
    given, entropy, ids, top = ref.logprobs(row, [1, 3, 4], 1.0, 3)
    assert np.allclose(given[:2], [np.log(0.4), -np.inf]) and np.isnan(given[2]) and ids.tolist() == [1, 2, 0]
    assert np.allclose(entropy, -(0.2 * np.log(0.2) + 0.8 * np.log(0.4))) and np.allclose(top, np.log([0.4, 0.4, 0.2]))
    assert ref.logprobs(np.array([0.0, np.nan]), [0], 1.0, 1)[2].tolist() == [-1]
