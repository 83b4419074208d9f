"""Host-side checks of the operators around the step: refusals come back with the documented codes before anything is
enqueued (fake pointers are never used), and the plain statements they are tested against hold by hand."""
import ctypes
import os
import subprocess
import sys
import types

import numpy as np
import pytest
import torch

import ops_reference as ref
from paper_2401_06706_b200 import binding, build, synth

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


@pytest.mark.parametrize("change,code", [({"head_dim": 96}, -10), ({"page_size": 8}, -10), ({"page_size": 48}, -10), ({"n_heads": 0}, -2),
                                         ({"n_pages": -1}, -2), ({"pages": None}, -1), ({"pages": FAKE + 8}, -7), ({"page_stride": 2 * 16 * 136 - 16}, -7),
                                         ({"page_stride": 2 * 16 * 136 + 8}, -7)])
def test_cache_refusals(lib, change, code):
    c = _cache(**change)
    assert lib.mcsd_append_kv(ctypes.byref(c), FAKE, 256, 128, FAKE, 256, 128, 1, 4, FAKE, None) == code
    assert lib.mcsd_read_kv(ctypes.byref(c), FAKE, 256, 128, FAKE, 256, 128, 1, 4, FAKE, None) == code
    assert lib.mcsd_gather_accepted_pages(ctypes.byref(c), 1, 0, FAKE, 4, 4, 2, FAKE, FAKE, FAKE, 3, None) == code


def test_row_call_refusals(lib):
    c = _cache()
    b = ctypes.byref(c)
    for f in (lib.mcsd_append_kv, lib.mcsd_read_kv):
        assert f(None, FAKE, 256, 128, FAKE, 256, 128, 1, 4, FAKE, None) == -1
        assert f(b, FAKE, 256, 128, FAKE, 256, 128, 3, 4, FAKE, None) == -3
        assert f(b, FAKE, 256, 128, FAKE, 256, 128, 1, -1, FAKE, None) == -2
        assert f(b, FAKE, -1, 128, FAKE, 256, 128, 1, 4, FAKE, None) == -7
        assert f(b, FAKE, 256, 128, FAKE, 256, 128, 1, 4, None, None) == -1
        assert f(b, None, 256, 128, None, 256, 128, 1, 0, None, None) == 0
    assert lib.mcsd_append_kv(b, None, 256, 128, FAKE, 256, 128, 1, 4, FAKE, None) == -1
    assert lib.mcsd_read_kv(b, None, 256, 128, None, 256, 128, 1, 4, FAKE, None) == -1
    assert lib.mcsd_read_kv(b, FAKE, 256, 127, FAKE, 256, 128, 1, 4, FAKE, None) == -7     # rows that overlap
    assert lib.mcsd_read_kv(b, FAKE, 100, 128, FAKE, 256, 128, 1, 4, FAKE, None) == -7


def test_gather_refusals(lib):
    c = _cache()
    call = lambda layers=1, stride=0, ld=4, width=4, batch=2, gamma=3, p=FAKE: lib.mcsd_gather_accepted_pages(
        ctypes.byref(c), layers, stride, p, ld, width, batch, FAKE, FAKE, FAKE, gamma, None)
    assert call(layers=-1) == -2 and call(batch=-1) == -2 and call(gamma=-1) == -2 and call(width=-1) == -2
    assert call(ld=3) == -7 and call(stride=8) == -7 and call(layers=2, stride=16) == -7 and call(p=None) == -1
    assert call(layers=0) == 0 and call(batch=0) == 0 and call(gamma=0) == 0


def test_kv_block_bytes(lib):
    assert binding.mcsd_kv_block_bytes(128, 16) == 16 * 136 and binding.mcsd_kv_block_bytes(64, 128) == 128 * 72
    for bad in ((0, 16), (32, 16), (256, 16), (128, 0), (128, 24), (128, 256), (-64, 16)):
        assert binding.mcsd_kv_block_bytes(*bad) == 0


def _attention(**kw):
    d = binding.McsdAttentionDesc()
    d.batch, d.n_nodes, d.n_heads, d.dtype, d.max_pages, d.ld_table = 2, 3, 4, 1, 8, 8
    d.q_seq_stride, d.q_node_stride, d.q_head_stride = 3 * 512, 512, 128
    d.out_seq_stride, d.out_node_stride, d.out_head_stride = 3 * 512, 512, 128
    d.scale, d.workspace, d.workspace_bytes = 0.1, FAKE, 1 << 40
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,code", [
    ({"batch": -1}, -2), ({"n_nodes": 0}, -2), ({"n_nodes": 513}, -10), ({"n_heads": 0}, -2), ({"n_heads": 5}, -2), ({"dtype": 0}, -3), ({"dtype": 7}, -3),
    ({"max_pages": -1}, -2), ({"ld_table": 7}, -7), ({"reserved": 1}, -2), ({"q_head_stride": -1}, -7), ({"out_head_stride": 127}, -7),
    ({"out_node_stride": 100}, -7), ({"out_seq_stride": 100}, -7), ({"scale": float("nan")}, -2), ({"scale": float("inf")}, -2), ({"workspace": None}, -8),
    ({"workspace": FAKE + 16}, -8), ({"workspace_bytes": 0}, -8), ({"max_pages": 1 << 27, "ld_table": 1 << 27}, -10)])
def test_attention_refusals(lib, change, code):
    parent = synth.tree_from_kconfig([2])
    c, d = _cache(), _attention(**change)
    assert lib.mcsd_tree_attention(ctypes.byref(d), ctypes.byref(c), FAKE, FAKE, parent.ctypes.data, FAKE, FAKE, None) == code


def test_attention_refuses_missing_pointers_and_bad_trees(lib):
    parent = synth.tree_from_kconfig([2])
    c, d = _cache(), _attention()
    call = lambda t=FAKE, p=FAKE, tree=parent.ctypes.data, q=FAKE, out=FAKE: lib.mcsd_tree_attention(
        ctypes.byref(d), ctypes.byref(c), t, p, tree, q, out, None)
    assert call(t=None) == -1 and call(p=None) == -1 and call(tree=None) == -1 and call(q=None) == -1 and call(out=None) == -1
    bad = np.array([-1, 1, 0], dtype=np.int32)
    assert call(tree=bad.ctypes.data) == -6
    assert lib.mcsd_tree_attention(None, ctypes.byref(c), FAKE, FAKE, parent.ctypes.data, FAKE, FAKE, None) == -1
    assert lib.mcsd_tree_attention(ctypes.byref(d), None, FAKE, FAKE, parent.ctypes.data, FAKE, FAKE, None) == -1
    assert lib.mcsd_tree_attention_workspace_bytes(ctypes.byref(d), ctypes.byref(c)) % 256 == 0
    assert lib.mcsd_tree_attention_workspace_bytes(None, ctypes.byref(c)) == 0
    d.n_heads = 3
    assert lib.mcsd_tree_attention_workspace_bytes(ctypes.byref(d), ctypes.byref(c)) == 0


def test_attention_workspace_is_sized_on_the_device_of_the_cache(lib, monkeypatch):
    """Its size depends on the device's multiprocessors, so the query runs where the calls will run, whatever is current."""
    where, asked = [], []

    class Guard:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            where.append(self.device)

        def __exit__(self, *exc):
            where.pop()

    class Lib:
        def __getattr__(self, name):
            return getattr(lib, name)

        def mcsd_tree_attention_workspace_bytes(self, d, c):
            asked.append(list(where))
            return lib.mcsd_tree_attention_workspace_bytes(d, c)

    monkeypatch.setattr(binding, "_on_device", Guard)
    monkeypatch.setattr(binding, "_settle", lambda device: None)
    monkeypatch.setattr(binding, "load_library", lambda path=None: Lib())
    cpu = torch.device("cpu")                        # (stands for the device of the cache)
    cache = types.SimpleNamespace(device=cpu, head_dim=128, page_size=16, n_heads=2, desc=_cache())
    att = binding.TreeAttention(2, synth.tree_from_kconfig([2]), 4, torch.bfloat16, cache, 8)
    assert asked == [[cpu]] and where == []


def _page_desc(**kw):
    d = binding.McsdPageDesc()
    d.batch, d.page_size, d.max_pages, d.ld_table, d.ring_capacity = 3, 16, 8, 8, 50
    d.start = d.page_table = d.held = d.ring = d.ring_state = FAKE
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("change,code", [
    ({"batch": -1}, -2), ({"batch": 4097}, -10), ({"page_size": 17}, -10), ({"max_pages": -1}, -2), ({"ld_table": 7}, -7), ({"new_tokens": -1}, -2),
    ({"ring_capacity": 0}, -2), ({"n_slots": -1}, -2), ({"reserved": 1}, -2), ({"start": None}, -1), ({"held": None}, -1), ({"ring": None}, -1),
    ({"ring_state": None}, -1), ({"page_table": None}, -1), ({"max_pages": 1 << 28, "ld_table": 1 << 28}, -10), ({"batch": 0}, 0)])
def test_page_table_refusals(lib, change, code):
    d = _page_desc(**change)
    assert lib.mcsd_build_page_tables(ctypes.byref(d)) == code
    assert lib.mcsd_build_page_tables(None) == -1


def _rules_call(lib, desc_kw=(), rule_kw=(), **kw):
    parent = synth.tree_from_kconfig([2])
    d, r = binding.McsdDesc(), binding.McsdLogitRules()
    d.batch, d.n_nodes, d.vocab, d.dtype = 2, 3, 64, 0
    for k, v in dict(desc_kw).items():
        setattr(d, k, v)
    for k, v in dict(rule_kw).items():
        setattr(r, k, v)
    a = dict(tree=parent.ctypes.data, cand=FAKE, logits=FAKE, ld_in=64, out=FAKE, ld_out=64, rows=3, begin=0, end=3)
    a.update(kw)
    return lib.mcsd_apply_logit_rules(ctypes.byref(d), ctypes.byref(r), a["tree"], a["cand"], a["logits"], a["ld_in"], a["out"], a["ld_out"],
                                      a["rows"], a["begin"], a["end"])


def test_logit_rule_refusals(lib):
    call = lambda *a, **k: _rules_call(lib, *a, **k)
    for kw, code in (({"vocab": 0}, -2), ({"vocab": 65537}, -10), ({"n_nodes": 0}, -2), ({"n_nodes": 513}, -10), ({"batch": -1}, -2), ({"batch": 65536}, -10),
                     ({"dtype": 5}, -3), ({"reserved": 2}, -2)):
        assert call(kw) == code, kw
    for kw, code in (({"n_bias": -1}, -2), ({"n_history": -1}, -2), ({"n_masks": -1}, -2), ({"masks": FAKE, "n_masks": 1, "ld_mask": 1}, -7),
                     ({"history": FAKE, "n_history": 4, "ld_history": 4}, -1), ({"history": FAKE, "history_len": FAKE, "n_history": 4, "ld_history": 3}, -7),
                     ({"bias_ids": FAKE, "n_bias": 2}, -1), ({"bias_values": FAKE, "n_bias": 2}, -1)):
        assert call((), kw) == code, kw
    assert call(ld_in=63) == -7 and call(ld_out=63) == -7 and call(logits=None) == -1 and call(out=None) == -1 and call(tree=None) == -1
    assert call(rows=4) == -2 and call(rows=-1) == -2 and call(begin=-1) == -2 and call(end=4) == -2 and call(begin=2, end=1) == -2
    assert call(ld_in=64, ld_out=72) == -7                                        # in place with two strides
    assert call((), {"repetition": FAKE}, cand=None) == -1
    assert call({"batch": 0}) == 0 and call(begin=1, end=1) == 0
    bad = np.array([-1, 1, 0], dtype=np.int32)
    assert call(tree=bad.ctypes.data) == -6
    assert lib.mcsd_apply_logit_rules(None, None, None, None, None, 0, None, 0, 0, 0, 0) == -1


def test_arrays_off_their_elements_are_refused(lib):
    """A kernel would fault on them: every device array of every call, one byte (or half an element) off."""
    b = ctypes.byref(_cache())
    for f in (lib.mcsd_append_kv, lib.mcsd_read_kv):
        for dtype, off in ((0, 2), (1, 1), (2, 1)):
            assert f(b, FAKE + off, 256, 128, FAKE, 256, 128, dtype, 4, FAKE, None) == -7
            assert f(b, FAKE, 256, 128, FAKE + off, 256, 128, dtype, 4, FAKE, None) == -7
        assert f(b, FAKE, 256, 128, FAKE, 256, 128, 1, 4, FAKE + 4, None) == -7
    for i in range(4):
        a = [FAKE + 2 * (i == j) for j in range(4)]
        assert lib.mcsd_gather_accepted_pages(b, 1, 0, a[0], 4, 4, 2, a[1], a[2], a[3], 3, None) == -7
    parent = synth.tree_from_kconfig([2])
    for i, off in enumerate((2, 2, 1, 1, 2)):
        a = [FAKE + off * (i == j) for j in range(5)]
        assert lib.mcsd_tree_attention(ctypes.byref(_attention()), b, a[0], a[1], parent.ctypes.data, a[2], a[3], a[4]) == -7
    for name in ("start", "count", "page_table", "held", "held_out", "ring", "ring_state", "ring_state_out", "cu_tokens", "status"):
        assert lib.mcsd_build_page_tables(ctypes.byref(_page_desc(**{name: FAKE + 2}))) == -7, name
    assert lib.mcsd_build_page_tables(ctypes.byref(_page_desc(slots=FAKE + 4, n_slots=5))) == -7
    for kw in ({"logits": FAKE + 2}, {"out": FAKE + 2}, {"cand": FAKE + 2}):
        assert _rules_call(lib, **kw) == -7, kw
    assert _rules_call(lib, {"dtype": 1}, logits=FAKE + 1) == -7 and _rules_call(lib, {"out_status": FAKE + 1}) == -7
    whole = dict(history=FAKE, history_len=FAKE, n_history=4, ld_history=4, bias_ids=FAKE, bias_values=FAKE, n_bias=1, masks=FAKE, n_masks=6, ld_mask=2)
    for name in ("history", "history_len", "prompt_len", "repetition", "frequency", "presence", "bias_ids", "bias_values", "masks", "mask_index"):
        assert _rules_call(lib, (), {**whole, name: FAKE + 2}) == -7, name


def test_trees_are_checked_without_an_allocation(lib, tmp_path):
    """No C++ exception reaches a C caller: a process whose `operator new` throws still gets its answer."""
    src, so = tmp_path / "no_new.cpp", tmp_path / "no_new.so"
    src.write_text("#include <cstdlib>\n#include <new>\nextern \"C\" int refuse_new = 0;\n"
                   "void *operator new(std::size_t n) { if (refuse_new) throw std::bad_alloc(); return std::malloc(n ? n : 1); }\n"
                   "void operator delete(void *p) noexcept { std::free(p); }\nvoid operator delete(void *p, std::size_t) noexcept { std::free(p); }\n")
    subprocess.run(["g++", "-shared", "-fPIC", "-O1", "-o", str(so), str(src)], check=True)
    code = f"""
import ctypes
new = ctypes.CDLL({str(so)!r}, mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL({binding.LIB_PATH!r})
parent = (ctypes.c_int32 * 5)(-1, 0, 0, 1, 3)
ctypes.c_int.in_dll(new, "refuse_new").value = 1
depth = lib.mcsd_tree_depth(parent, 5)
ctypes.c_int.in_dll(new, "refuse_new").value = 0
print("depth", depth)
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, env={**os.environ, "LD_PRELOAD": str(so)})
    assert r.returncode == 0 and r.stdout.strip() == "depth 3", (r.returncode, r.stdout, r.stderr[-500:])


def test_status_bits_match_the_header():
    text = open(os.path.join(build.ROOT, "include", "mcsd.h")).read()
    for name, value in (("NO_PAGES", binding.STATUS_NO_PAGES), ("BAD_MASK", binding.STATUS_BAD_MASK)):
        assert f"#define MCSD_STATUS_{name} {value}" in text
    assert f"#define MCSD_MAX_SEQUENCES {binding.MAX_SEQUENCES}" in text


# ---------------------------------------------------------------- the plain statements, by hand
def test_reference_rules_by_hand():
    parent = np.array([-1, 0, 0, 1], dtype=np.int32)
    logits = np.array([[[2.0, -1.0, 0.5, 4.0]] * 4])
    cand = np.array([[3, 1, 2, 1]])
    out, _, _ = ref.logit_rules(logits, parent, cand, history=np.array([[0, 1, 3]]), history_len=[3], prompt_len=[1], repetition=[2.0], frequency=[0.5],
                                presence=[0.25], bias_ids=np.array([[2, 2]]), bias_values=np.array([[9.0, 1.0]]))
    assert np.allclose(out[0, 0], [1.0, -2.75, 1.5, 1.25])           # prompt 0; generated 1 and 3 once each; bias on 2
    assert np.allclose(out[0, 1], [1.0, -3.25, 1.5, 1.25])           # node 1 adds token 1
    assert np.allclose(out[0, 2], [1.0, -2.75, 0.25 - 0.75 + 1, 1.25])
    assert np.allclose(out[0, 3], [1.0, -3.75, 1.5, 1.25])           # token 1 at nodes 1 and 3


def test_reference_pages_by_hand():
    table = np.array([[7, -1], [5, 6], [-1, -1]])
    got = ref.page_tables(np.array([16, 0, 0]), np.array([1, 3, 17]), table, np.array([1, 2, 0]), np.array([0, 1, 2, 3, 4, 9, 9, 9]), 1, 4, 16)
    assert got[0].tolist() == [[7, 1], [5, 6], [2, 3]] and got[1].tolist() == [2, 1, 2]
    assert got[2].tolist() == [0, 1, 2, 3, 4, 6, 9, 9] and got[3:5] == (4, 2)
    assert got[5].tolist() == [16] + [80, 81, 82] + [32 + i for i in range(16)] + [48] and got[7].tolist() == [0, 0, 0]


def test_reference_quantiser_by_hand():
    x = np.array([[0.0, 15.0, 7.0, 7.5], [2.0, 2.0, 2.0, 2.0], [np.inf, 0, 0, 0]])
    codes, scale, mid = ref.quantise(x)
    assert scale.tolist()[:2] == [1.0, 0.0] and mid.tolist()[:2] == [8.0, 2.0] and np.isnan(mid[2]) and scale[2] == 0
    assert codes[0].tolist() == [0, 15, 7, 8] and codes[1].tolist() == [8] * 4     # 7.5: a tie, to the even -0 -> 8


def test_reference_attention_by_hand():
    """Two keys of the prefix and a tree of three nodes: node 1 and node 2 do not see each other."""
    ps, D = 16, 64
    pages = np.zeros((1, 1, ps * (D + 8)), dtype=np.uint8)
    rng = np.random.default_rng(0)
    k, v = rng.standard_normal((5, 1, D)), rng.standard_normal((5, 1, D))
    pages = ref.append(pages, k, v, np.arange(5), D, ps)
    q = rng.standard_normal((1, 3, 1, D))
    out, lse, _, _ = ref.attention(q, pages, np.array([[0]]), np.array([2]), [-1, 0, 0], D, ps, 0.125, 2.0 ** -10)
    kk, vv = (np.stack([ref.row_values(pages, 0, t, D, ps)[i][0] for t in range(5)]) for i in (0, 1))
    for n, see in enumerate(([0, 1, 2], [0, 1, 2, 3], [0, 1, 2, 4])):
        s = 0.125 * kk[see] @ q[0, n, 0]
        w = np.exp(s) / np.exp(s).sum()
        assert np.allclose(out[0, n, 0], w @ vv[see]) and np.allclose(lse[0, n, 0], np.log(np.exp(s).sum()))
