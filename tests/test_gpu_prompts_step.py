"""The operators of prompts and long conversations together, as a serving loop uses them: prompts in chunks (page tables, append, attention,
weights), eviction, the pages that became free, decoding on what is left, verified paths with their log probabilities; captured; expired waits."""
import numpy as np
import pytest
import torch

import ops_reference as ops
import prompts_reference as ref
from gpu_util import library_options
from paper_2401_06706_b200 import binding, synth
from prompts_util import attend, attention, check_attention, host, problem

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


def test_a_serving_loop_over_long_conversations():
    g = torch.Generator().manual_seed(21)
    B, ps, D, kv, heads, layers, W, n_pages = 4, 16, 64, 2, 6, 2, 30, 110
    budget, sink, recent, dt = 120, 4, 20, torch.bfloat16
    cache = binding.KvCache.empty(n_pages, kv, D, ps, n_layers=layers)
    weights = torch.full((layers, n_pages, kv, ps), float("nan"), device="cuda")       # (a row's weight begins with its own chunk)
    plan = binding.PageTables.empty(B, W, n_pages, ps)
    att = binding.ChunkAttention(B, 700, heads, dt, cache.layer(0), W, max_new=260)
    small = binding.ChunkAttention(B, 3 * B, heads, dt, cache.layer(0), W, max_new=3)
    length = torch.zeros(B, **I32)

    def chunk(call, counts, last):
        """New tokens of every sequence through all layers, each call against its statement."""
        count = torch.tensor(counts, **I32)
        T = sum(counts)
        slots = torch.empty(T, dtype=torch.int64, device="cuda")
        plan.mcsd_build_page_tables(length, count, slots=slots)
        assert (plan.status == 0).all() and (slots >= 0).all()
        for l in range(layers):
            layer = cache.layer(l)
            k, v = (torch.randn((T, kv, D), generator=g).to(dt).cuda() for _ in range(2))
            binding.mcsd_append_kv(layer, k, v, slots)
            q = torch.randn((T, heads, D), generator=g).to(dt).cuda()
            r = call.mcsd_chunk_attention(q, layer, plan.table, length, plan.cu_tokens)
            before = weights[l].clone()
            call.mcsd_accumulate_weights(q, r.lse, layer, plan.table, length, plan.cu_tokens, weights[l], decay=0.5, last_tokens=last)
            args = (layer.pages.cpu().numpy(), host(plan.table), host(length), host(plan.cu_tokens))
            want, lse, tol, tol_lse = ref.chunk_attention(host(q), *args, call.max_new, D, ps, D ** -0.5, torch.finfo(dt).eps)
            assert (np.abs(host(r.out) - want) <= tol).all() and (np.abs(host(r.lse) - lse) <= tol_lse).all()
            w, tol = ref.accumulate(host(q), host(r.lse), args[0], host(before), *args[1:], call.max_new, D, ps, D ** -0.5, 0.5, last)
            got = host(weights[l])
            assert ((np.abs(got - w) <= tol) | (np.isnan(got) & np.isnan(w))).all()
        length.add_(count)

    chunk(att, [200, 1, 90, 33], 16)
    chunk(att, [250, 130, 1, 0], 16)
    for turn in range(3):
        # the conversations that are too long are cut, every layer and head by its own weights
        pages, w, before = cache.pages.cpu().numpy(), weights.cpu().numpy(), host(length)
        new_len = binding.mcsd_evict_rows(cache, weights, plan.table, length, budget, sink=sink, recent=recent)
        want = ref.evict(pages, w, host(plan.table), before, [budget] * B, sink, recent, D, ps)
        assert np.array_equal(cache.pages.cpu().numpy(), want[0]) and np.array_equal(weights.cpu().numpy().view(np.uint32), want[1].view(np.uint32))
        assert np.array_equal(host(new_len), want[2]) and (host(new_len) <= budget).all()
        free = int(plan.ring_state[1])
        held = plan.held.clone()
        plan.mcsd_build_page_tables(new_len, 0)          # (no new tokens: surplus pages go back)
        assert int(plan.ring_state[1]) == free + int((held - plan.held).sum())
        length.copy_(new_len)
        chunk(small, [1, 3, 2, 1], 0)                    # decoding
        chunk(att, [7, 0, 150, 40 * turn], 0)


def test_prompt_and_path_log_probabilities_in_a_step():
    """Prompt tokens against the rows before them; then candidates drawn, verified, and the walk's tokens reported under the same logit rules."""
    g = torch.Generator().manual_seed(22)
    parent = synth.tree_from_kconfig([3, 2, 1])
    N, B, V, dt = len(parent), 6, 900, torch.float16
    n_int = binding._n_internal(parent)
    prompt = torch.randint(0, V, (40,), generator=g, dtype=torch.int32).cuda()
    logits = (2 * torch.randn((40, V), generator=g)).to(dt).cuda()
    scorer = binding.TokenLogprobs(64, V, dt, n_top=3)
    r = scorer.mcsd_token_logprobs(logits, torch.roll(prompt, -1), row_index=torch.arange(40, **I32) - (torch.arange(40, **I32) == 39).int() * 100)
    for i in range(39):
        given, entropy, ids, top = ref.logprobs(host(logits[i]), [int(prompt[i + 1])], 1.0, 3)
        assert abs(float(r.logprobs[i]) - given[0]) < 1e-5 and np.array_equal(host(r.top_ids[i]), ids) and abs(float(r.entropy[i]) - entropy) < 1e-5
    assert float(r.logprobs[39]) == 0
    target = (2 * torch.randn((B, N, V), generator=g)).to(dt).cuda()
    draft = (target[:, :n_int].float() + 0.5 * torch.randn((B, n_int, V), generator=g).cuda()).to(dt)
    cand = torch.full((B, N), -1, **I32)
    cand[:, 0] = 5
    binding.mcsd_sample_candidates(draft, parent, torch.rand((B, N), generator=g).clamp(1e-3, 1 - 1e-3).cuda(), 1.0, 1, node_begin=0, node_end=n_int, cand=cand)
    rules = binding.LogitRules(bias_ids=torch.tensor([[7, 9]] * B, **I32), bias_values=torch.tensor([[-1e4, 2.0]] * B, device="cuda"))
    binding.mcsd_apply_logit_rules(target, parent, cand, rules)
    ver = binding.Verifier(B, parent, V, dt)
    paths = binding.TokenLogprobs(B * 4, V, dt, n_top=5)
    unif = torch.rand((B, N, 2), generator=g).cuda()

    def step():
        out = ver.mcsd_verify(target, draft, cand, unif, 1.0, 1)
        return out, paths.mcsd_path_logprobs(target, out.path_nodes, out.tokens)

    out, r = step()
    torch.cuda.synchronize()
    for b in range(B):
        for j in range(int(out.accept_len[b]) + 1):
            node = 0 if j == 0 else int(out.path_nodes[b, j - 1])
            given, _, ids, _ = ref.logprobs(host(target[b, node]), [int(out.tokens[b, j])], 1.0, 5)
            assert abs(float(r.logprobs[b, j]) - given[0]) < 2e-5 and np.array_equal(host(r.top_ids[b, j]), ids) and 7 not in ids
    want = [t.clone() for t in (out.tokens, r.logprobs, r.top_ids)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    paths.logprobs.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (out.tokens, r.logprobs, r.top_ids)))


def test_a_captured_prompt_step():
    """Page tables, append, attention, weights, eviction and the return of pages in one graph, replayed on what the replay before left, against
    the same calls one by one."""
    g = torch.Generator().manual_seed(23)
    B, ps, D, kv, heads, W, n_pages, T = 3, 16, 128, 2, 8, 24, 80, 3 * 70
    dt = torch.bfloat16
    new = {k: torch.empty((T, h, D), dtype=dt, device="cuda") for k, h in (("q", heads), ("k", kv), ("v", kv))}

    def make():
        cache = binding.KvCache.empty(n_pages, kv, D, ps)
        return dict(cache=cache, plan=binding.PageTables.empty(B, W, n_pages, ps), att=binding.ChunkAttention(B, T, heads, dt, cache, W, max_new=70),
                    weights=torch.zeros((n_pages, kv, ps), device="cuda"), length=torch.zeros(B, **I32), slots=torch.empty(T, dtype=torch.int64, device="cuda"),
                    cut=torch.zeros(B, **I32))

    def step(s):
        s["plan"].mcsd_build_page_tables(s["length"], 70, slots=s["slots"])
        binding.mcsd_append_kv(s["cache"], new["k"], new["v"], s["slots"])
        r = s["att"].mcsd_chunk_attention(new["q"], s["cache"], s["plan"].table, s["length"], s["plan"].cu_tokens)
        s["att"].mcsd_accumulate_weights(new["q"], r.lse, s["cache"], s["plan"].table, s["length"], s["plan"].cu_tokens, s["weights"], decay=0.9)
        s["length"].add_(70)
        binding.mcsd_evict_rows(s["cache"], s["weights"], s["plan"].table, s["length"], 150, sink=4, recent=30, len_out=s["cut"])
        s["plan"].mcsd_build_page_tables(s["cut"], 0)
        s["length"].copy_(s["cut"])
        return r.out

    one, two = make(), make()
    scratch = make()
    for t in new.values():
        t.normal_()
    step(scratch)                                    # (looks up launch attributes)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(two)
    for i in range(5):
        for t in new.values():
            t.copy_(torch.randn(t.shape, generator=g))
        want = step(one)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.isfinite(out).all()
        for a, b in ((one["cache"].pages, two["cache"].pages), (one["weights"], two["weights"]), (one["length"], two["length"]), (one["plan"].table, two["plan"].table)):
            assert torch.equal(a, b)
    assert (one["length"] == 150).all()


def test_new_objects_are_ready_for_any_stream():
    """Objects made while their stream is busy, used on another stream at once: nothing enqueued for making them comes after the call."""
    p = problem(24, [100, 20], [40, 3], 4, 2, 64, 16, torch.bfloat16)
    want = attend(p)
    logits = torch.randn((8, 500), device="cuda")
    tokens = torch.arange(8, **I32)
    ref_lp = binding.TokenLogprobs(8, 500, torch.float32, n_top=2).mcsd_token_logprobs(logits, tokens).logprobs.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(20_000_000)                    # about 10 ms on the current stream
    a = attention(p)
    torch.cuda._sleep(20_000_000)
    c = binding.TokenLogprobs(8, 500, torch.float32, n_top=2)
    with torch.cuda.stream(side):
        r = a.mcsd_chunk_attention(p.q, p.cache, p.table, p.start, p.cu)
        lp = c.mcsd_token_logprobs(logits, tokens)
    torch.cuda.synchronize()
    assert torch.equal(r.out, want.out) and torch.equal(r.lse, want.lse) and torch.equal(lp.logprobs, ref_lp)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("starts", [[40, -1, 3], [3000, -1, 700]])
def test_expired_waits_give_nan_and_return(D, starts):
    """The kernels whose roles wait for one another: a barrier expects an arrival that never comes, the waits run out, all roles go on to their
    end, rows of used entries are NaN (of blocks in one piece and of divided ones), and so are the weights."""
    p = problem(25, starts, [90, 0, 150], 4, 2, D, 16, torch.bfloat16)
    a = attention(p)
    r = a.mcsd_chunk_attention(p.q, p.cache, p.table, p.start, p.cu)
    w = torch.zeros((p.cache.n_pages, 2, 16), device="cuda")
    a.mcsd_accumulate_weights(p.q, r.lse, p.cache, p.table, p.start, p.cu, w)
    out, lse, weights = r.out.clone(), r.lse.clone(), w.clone()
    torch.cuda.synchronize()
    with library_options(wait_polls=4, test_extra_tx=16):
        a.mcsd_chunk_attention(p.q, p.cache, p.table, p.start, p.cu)
        w.zero_()
        a.mcsd_accumulate_weights(p.q, lse, p.cache, p.table, p.start, p.cu, w)
        torch.cuda.synchronize()                     # (it returned)
    assert torch.isnan(a.out).all() and torch.isnan(a.lse).all()
    assert torch.isnan(w[weights != 0]).all() and (w[weights == 0] == 0).all()
    # the library and the context are as usable as before
    a.mcsd_chunk_attention(p.q, p.cache, p.table, p.start, p.cu)
    w.zero_()
    a.mcsd_accumulate_weights(p.q, lse, p.cache, p.table, p.start, p.cu, w)
    torch.cuda.synchronize()
    assert torch.equal(a.out, out) and torch.equal(a.lse, lse) and torch.equal(w, weights)
    check_attention(p, r)
