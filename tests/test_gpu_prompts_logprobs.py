"""mcsd_token_logprobs against a plain statement in 64 bits."""
import numpy as np
import pytest
import torch

import prompts_reference as ref
from paper_2401_06706_b200 import binding, synth
from prompts_util import host

pytestmark = pytest.mark.gpu
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _check(logits, tokens, r, temperature, n_top, rows=None):
    """Rows of outputs against the statement. What float32 may do: a scaled logit is off by 2^-23 of its distance from the largest one (two
    roundings), a sum of exponentials by that of its terms and 2^-20 for the approximations and the order, its logarithm and the result by
    a step each."""
    l, t = host(logits), tokens.cpu().numpy().reshape(tokens.shape[0], -1)
    lp, en = host(r.logprobs).reshape(t.shape).astype(np.float64), host(r.entropy).astype(np.float64)
    ids, tl = host(r.top_ids), host(r.top_logprobs).astype(np.float64)
    for i in range(t.shape[0]) if rows is None else rows:
        given, entropy, want, top = ref.logprobs(l[i], t[i], temperature, n_top)
        assert np.array_equal(ids[i], want), (i, ids[i], want)
        finite = l[i][np.isfinite(l[i])]
        span = (finite.max() - finite.min()) / temperature if finite.size else 0.0
        slack = lambda x: 2.0 ** -19 + 2.0 ** -22 * (np.abs(np.where(np.isfinite(x), x, 0)) + np.log(len(l[i])))
        for got, w, tol in ((lp[i], given, slack(given)), (tl[i], top, slack(top)), (en[i:i + 1], np.array([entropy]), np.array([2.0 ** -18 + 2.0 ** -21 * min(span, 100)]))):
            with np.errstate(invalid="ignore"):
                ok = (np.abs(got - w) <= tol) | (got == w) | (np.isnan(got) & np.isnan(w))
            assert ok.all(), (i, got, w, tol)


def _run(logits, tokens, temperature=1.0, n_top=5, **kw):
    n_given = 1 if tokens.dim() == 1 else tokens.shape[1]
    c = binding.TokenLogprobs(tokens.shape[0], logits.shape[-1], logits.dtype, n_given=n_given, n_top=n_top)
    r = c.mcsd_token_logprobs(logits, tokens, temperature=temperature, **kw)
    torch.cuda.synchronize()
    return r


def _logits(seed, rows, V, dtype, scale=2.5):
    return (scale * torch.randn((rows, V), generator=torch.Generator().manual_seed(seed))).to(dtype).cuda()


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("V", [1, 2, 7, 33, 255, 1000, 4097, 32000, 50272, 65536])
@pytest.mark.parametrize("n_top", [0, 1, 5, 32])
def test_against_reference(dtype, V, n_top):
    n_top = min(n_top, V)
    logits = _logits(V + n_top, 6, V, DTYPES[dtype])
    tokens = torch.randint(0, V, (6,), generator=torch.Generator().manual_seed(V), dtype=torch.int32).cuda()
    for T in (1.0, 0.6):
        _check(logits, tokens, _run(logits, tokens, T, n_top), T, n_top)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("V", [40, 3001, 32000])
def test_orders_that_are_hard_to_select_from(dtype, V):
    """Rising and falling rows, rows of one value, of two, largest tokens side by side or in one thread's elements, zeros of both signs."""
    base = torch.arange(V).float()
    step = 64.0 / V
    rows = [base * step, -base * step, torch.zeros(V), (base % 2), torch.where(base % 2 == 0, 0.0, -0.0), torch.where(base >= V - 20, 3.0, 0.0),
            torch.where(base < 20, 3.0, 1.0), torch.where(base % 64 == 5, 9.0, base * 0), torch.where(base % 1024 < 8, base * step, -50.0), (base * 7919) % V * step]
    logits = torch.stack(rows).to(DTYPES[dtype]).cuda()
    tokens = torch.randint(0, V, (len(rows),), generator=torch.Generator().manual_seed(V), dtype=torch.int32).cuda()
    for n_top in (1, 20, 32):
        _check(logits, tokens, _run(logits, tokens, 1.0, n_top), 1.0, n_top)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_masked_infinite_and_nan_rows(dtype):
    V = 5000
    logits = _logits(3, 9, V, DTYPES[dtype])
    logits[0, 7:] = -np.inf                          # fewer tokens left than alternatives asked for
    logits[1, :] = -np.inf
    logits[2, 4321] = float("nan")
    logits[3, 17] = np.inf
    logits[4, ::2] = -np.inf
    logits[5] = torch.finfo(logits.dtype).min        # every token masked by the lowest value: all equal
    logits[6, 1:] = torch.finfo(logits.dtype).min
    logits[7, :] = -np.inf
    logits[7, 4999] = 2.0
    logits[8, 11] = -float("nan")
    tokens = torch.tensor([3, 0, 1, 17, 2, 9, 0, 4999, 5], dtype=torch.int32, device="cuda")
    _check(logits, tokens, _run(logits, tokens, 1.0, 20), 1.0, 20)


@pytest.mark.parametrize("temperature", [0.01, 0.3, 5.0, 1000.0])
def test_temperatures(temperature):
    logits = _logits(4, 5, 32000, torch.float32, 8.0)
    logits[4] *= 20
    tokens = torch.randint(0, 32000, (5,), generator=torch.Generator().manual_seed(4), dtype=torch.int32).cuda()
    _check(logits, tokens, _run(logits, tokens, temperature, 8), temperature, 8)


def test_several_tokens_a_row_and_tokens_that_are_not_there():
    logits = _logits(5, 4, 1234, torch.bfloat16)
    tokens = torch.randint(0, 1234, (4, 300), generator=torch.Generator().manual_seed(5), dtype=torch.int32)
    tokens[0, 3], tokens[1, 7], tokens[2, 299] = -1, 1234, 2**31 - 1
    _check(logits, tokens.cuda(), _run(logits, tokens.cuda(), 0.9, 3), 0.9, 3)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("pad,off", [(0, 0), (8, 0), (3, 0), (5, 1)])
def test_strided_rows(dtype, pad, off):
    """Rows inside a larger tensor, at offsets off 16 bytes; a row index that repeats rows and names some that are not there."""
    V, R = 4099, 7
    full = torch.full((R, V + pad + off), 1e4, device="cuda").to(DTYPES[dtype])
    rows = _logits(6, R, V, DTYPES[dtype])
    full[:, off:off + V] = rows
    index = torch.tensor([6, 0, 0, -1, 3, 7, 2**31 - 1, 5], dtype=torch.int32, device="cuda")
    tokens = torch.randint(0, V, (8,), generator=torch.Generator().manual_seed(6), dtype=torch.int32).cuda()
    c = binding.TokenLogprobs(8, V, DTYPES[dtype], n_top=4)
    for t in (c.logprobs, c.entropy, c.top_ids, c.top_logprobs):
        t.fill_(77)
    r = c.mcsd_token_logprobs(full[:, off:off + V], tokens, row_index=index)
    torch.cuda.synchronize()
    there = (index >= 0) & (index < R)
    for t in (r.logprobs, r.entropy, r.top_ids, r.top_logprobs):
        assert (t[~there] == 77).all()
    _check(rows[index.clamp(0, R - 1).long()], tokens, r, 1.0, 4, rows=torch.nonzero(there)[:, 0].tolist())


def test_many_rows():
    """More rows than CTAs are resident at once."""
    logits = _logits(7, 5000, 300, torch.float16)
    tokens = torch.randint(0, 300, (5000,), generator=torch.Generator().manual_seed(7), dtype=torch.int32).cuda()
    r = _run(logits, tokens, 1.0, 3)
    _check(logits, tokens, r, 1.0, 3, rows=list(range(0, 5000, 83)) + [4999])
    want = torch.log_softmax(logits.double(), -1)
    assert (r.logprobs.double() - want.gather(1, tokens.long()[:, None])[:, 0]).abs().max() < 1e-5


def test_rows_beyond_four_gigabytes():
    V, R = 65536, 17000                              # 4.4 GB of bf16 logits
    logits = torch.zeros((R, V), dtype=torch.bfloat16, device="cuda")
    logits[-3:] = _logits(8, 3, V, torch.bfloat16)
    index = torch.tensor([R - 1, 0, R - 3], dtype=torch.int32, device="cuda")
    tokens = torch.tensor([5, 65535, 777], dtype=torch.int32, device="cuda")
    r = _run(logits, tokens, 1.0, 6, row_index=index)
    _check(logits[index.long()], tokens, r, 1.0, 6)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_paths_of_a_verification(dtype):
    """mcsd_verify's walks: each of their tokens against the row it was drawn from, entries behind a walk's end left alone; captured too."""
    w = synth.Workload("paths", 12, 3000, "3x2x1", dtype, "normal", 2.0, 1.0, 1.0, 1.0, 1, 9)
    inp = synth.make_inputs(w, "cuda:0")
    v = binding.Verifier(w.batch, inp.parent, w.vocab, synth.TORCH_DTYPES[w.dtype], "cuda:0")
    out = v.mcsd_verify(inp.target, inp.draft, inp.cand, inp.unif, w.temperature, w.mode)
    c = binding.TokenLogprobs(out.tokens.numel(), w.vocab, inp.target.dtype, n_top=4)
    r = c.mcsd_path_logprobs(inp.target, out.path_nodes, out.tokens, temperature=0.8)
    torch.cuda.synchronize()
    accept, nodes, tokens = host(out.accept_len), host(out.path_nodes), host(out.tokens)
    written = 0
    for b in range(w.batch):
        for j in range(tokens.shape[1]):
            if j > accept[b]:
                assert (r.logprobs[b, j] == 0) and (r.entropy[b, j] == 0) and (r.top_ids[b, j] == 0).all() and (r.top_logprobs[b, j] == 0).all()
                continue
            node = 0 if j == 0 else nodes[b, j - 1]
            given, entropy, ids, top = ref.logprobs(host(inp.target[b, node]), [tokens[b, j]], 0.8, 4)
            assert abs(float(r.logprobs[b, j]) - given[0]) < 1e-5 and abs(float(r.entropy[b, j]) - entropy) < 2e-5
            assert np.array_equal(host(r.top_ids[b, j]), ids) and np.abs(host(r.top_logprobs[b, j]) - top).max() < 1e-5
            written += 1
    assert written > w.batch
    keep = [t.clone() for t in (r.logprobs, r.entropy, r.top_ids, r.top_logprobs)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.mcsd_path_logprobs(inp.target, out.path_nodes, out.tokens, temperature=0.8)
    for t in (c.logprobs, c.entropy, c.top_ids, c.top_logprobs):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(keep, (r.logprobs, r.entropy, r.top_ids, r.top_logprobs)))


def test_outputs_are_optional():
    logits = _logits(9, 3, 900, torch.float16)
    tokens = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    want = _run(logits, tokens, 1.0, 4)
    for drop in ("logprobs", "entropy", "top_ids", "top_logprobs"):
        c = binding.TokenLogprobs(3, 900, torch.float16, n_top=4)
        setattr(c.desc, drop, None)
        r = c.mcsd_token_logprobs(logits, tokens)
        for name in ("logprobs", "entropy", "top_ids", "top_logprobs"):
            assert torch.equal(getattr(r, name), torch.zeros_like(getattr(r, name)) if name == drop else getattr(want, name)), (drop, name)
