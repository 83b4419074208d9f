"""The operators together, as a serving loop uses them: admission of prompts, then steps of page tables, append of the
tree's rows, tree attention, logit rules, verification, and the move of the accepted rows."""
import numpy as np
import pytest
import torch

import ops_reference as ref
from paper_2401_06706_b200 import binding, synth

pytestmark = pytest.mark.gpu


def test_serving_loop():
    g = torch.Generator().manual_seed(11)
    parent = synth.tree_from_kconfig([3, 2, 1])
    N, B, V, ps, D, kv, heads, layers = len(parent), 5, 700, 16, 64, 2, 4, 2
    n_int = binding._n_internal(parent)
    dt = torch.bfloat16
    cache = binding.KvCache.empty(60, kv, D, ps, n_layers=layers)
    plan = binding.PageTables.empty(B, 12, 60, ps)
    i32 = dict(dtype=torch.int32, device="cuda")

    # what the model would hand over, by (sequence, position): kept here to check the cache against
    truth = [[None] * 12 * ps for _ in range(B)]

    def rows(n):
        return torch.randn((layers, 2, n, kv, D), generator=g).to(dt)

    def store(seq_pos, x, slots):
        for l in range(layers):
            binding.mcsd_append_kv(cache.layer(l), x[l, 0].cuda(), x[l, 1].cuda(), slots)
        for i, (b, t) in enumerate(seq_pos):
            truth[b][t] = x[:, :, i]

    # prompts of different lengths
    lengths = [70, 1, 16, 33, 50]
    slots = torch.empty(sum(lengths), dtype=torch.int64, device="cuda")
    plan.mcsd_build_page_tables(torch.zeros(B, **i32), torch.tensor(lengths, **i32), slots=slots)
    store([(b, t) for b in range(B) for t in range(lengths[b])], rows(sum(lengths)), slots)
    prefix = torch.tensor(lengths, **i32)
    history = torch.randint(0, V, (B, 200), generator=g, dtype=torch.int32).cuda()
    rules = binding.LogitRules(history=history, history_len=prefix, prompt_len=torch.tensor(lengths, **i32), repetition=torch.full((B,), 1.2, device="cuda"),
                               presence=torch.full((B,), 0.3, device="cuda"))
    att = binding.TreeAttention(B, parent, heads, dt, cache.layer(0), 12)
    ver = binding.Verifier(B, parent, V, dt)
    tree_slots = torch.empty(B * N, dtype=torch.int64, device="cuda")
    for step in range(4):
        plan.mcsd_build_page_tables(prefix, N, slots=tree_slots)
        assert (plan.status == 0).all()
        start = prefix.tolist()
        store([(b, start[b] + n) for b in range(B) for n in range(N)], rows(B * N), tree_slots)
        for l in range(layers):
            q = torch.randn((B, N, heads, D), generator=g).to(dt).cuda()
            r = att.mcsd_tree_attention(q, cache.layer(l), plan.table, prefix)
            want, _, tol, _ = ref.attention(q.float().cpu().numpy(), cache.layer(l).pages.cpu().numpy(), plan.table.cpu().numpy(),
                                            prefix.cpu().numpy(), parent, D, ps, D ** -0.5, torch.finfo(dt).eps)
            assert (np.abs(r.out.float().cpu().numpy() - want) <= tol).all()
        target = (2 * torch.randn((B, N, V), generator=g)).to(dt).cuda()
        draft = (target[:, :n_int].float() + 0.5 * torch.randn((B, n_int, V), generator=g).cuda()).to(dt)
        draft_kept, target_kept = draft.clone(), target.clone()
        cand = torch.full((B, N), -1, **i32)
        cand[:, 0] = history[torch.arange(B), prefix.long() - 1]
        unif = torch.rand((B, N), generator=g).clamp(1e-3, 1 - 1e-3).cuda()
        level = 0
        while level < n_int:                         # the draft model level by level, under the rules
            kids = [n for n in range(N) if parent[n] == level]
            binding.mcsd_apply_logit_rules(draft, parent, cand, rules, node_begin=level, node_end=level + 1)
            binding.mcsd_sample_candidates(draft, parent, unif, 1.0, 1, node_begin=level, node_end=level + 1, cand=cand)
            assert (cand[:, kids] >= 0).all()
            level += 1
        binding.mcsd_apply_logit_rules(target, parent, cand, rules)
        kw = dict(history=history.cpu().numpy(), history_len=prefix.cpu().numpy(), prompt_len=np.array(lengths), repetition=np.full(B, np.float32(1.2)),
                  presence=np.full(B, np.float32(0.3)))
        for got, raw in ((target, target_kept), (draft, draft_kept)):
            want, size, _ = ref.logit_rules(raw.float().cpu().numpy(), parent, cand.cpu().numpy(), **kw)
            assert (np.abs(got.float().cpu().numpy() - want) <= torch.finfo(dt).eps / 2 * np.abs(want) + 2.0 ** -22 * size).all()
        out = ver.mcsd_verify(target, draft, cand, torch.rand((B, N, 2), generator=g).cuda(), 1.0, 1)
        binding.mcsd_gather_accepted_pages(cache, plan.table, prefix, out.path_nodes, out.accept_len)
        accept, nodes = out.accept_len.tolist(), out.path_nodes.tolist()
        for b in range(B):
            kept = [truth[b][start[b] + nodes[b][i]] for i in range(accept[b])]
            for i, x in enumerate(kept):
                truth[b][start[b] + 1 + i] = x
            n = accept[b] + 1
            history[b, start[b]:start[b] + n] = out.tokens[b, :n]
        prefix += out.accept_len + 1
        # every committed position of every layer still reads as the row that belongs there
        for b in range(B):
            n = int(prefix[b]) - 1                   # (the last token's row comes with the next tree)
            pos = torch.arange(n, device="cuda")
            at = plan.table[b, pos // ps].long() * ps + pos % ps
            want = torch.stack([truth[b][t] for t in range(n)], 2).cuda()
            fresh = binding.KvCache.empty(-(-n // ps), kv, D, ps)
            for l in range(layers):
                binding.mcsd_append_kv(fresh, want[l, 0].contiguous(), want[l, 1].contiguous(), pos)
                a, c = binding.mcsd_read_kv(cache.layer(l), at), binding.mcsd_read_kv(fresh, pos)
                assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])
    # one request ends: its pages go back, the others keep theirs
    free = int(plan.ring_state[1])
    held = plan.held.clone()
    done = torch.full((B,), -1, **i32)
    done[2] = 0
    plan.mcsd_build_page_tables(done, 0)
    assert int(plan.ring_state[1]) == free + int(held[2]) and int(plan.held[2]) == 0
    assert torch.equal(plan.held[[0, 1, 3, 4]], held[[0, 1, 3, 4]])


def test_a_captured_step():
    """A whole step (page tables, append and attention in two layers, rules and sampler level by level, verification, move of the
    accepted rows, read back, lengths and history advanced) captured in one graph and replayed: every part against its statement
    on what the replay before left."""
    g = torch.Generator().manual_seed(12)
    parent = synth.tree_from_kconfig([3, 2, 1])
    N, B, V, ps, D, kv, heads, layers, W, n_pages = len(parent), 4, 500, 16, 64, 2, 4, 2, 14, 64
    n_int, dt, gamma = binding._n_internal(parent), torch.bfloat16, 3
    i32 = dict(dtype=torch.int32, device="cuda")
    cache = binding.KvCache.empty(n_pages, kv, D, ps, n_layers=layers)
    plan = binding.PageTables.empty(B, W, n_pages, ps)
    lengths = [70, 1, 15, 40]
    slots = torch.empty(sum(lengths), dtype=torch.int64, device="cuda")
    plan.mcsd_build_page_tables(torch.zeros(B, **i32), torch.tensor(lengths, **i32), slots=slots)
    for l in range(layers):
        x = torch.randn((2, sum(lengths), kv, D), generator=g).to(dt).cuda()
        binding.mcsd_append_kv(cache.layer(l), x[0], x[1], slots)
    prefix, prompt = torch.tensor(lengths, **i32), torch.tensor(lengths, **i32)
    history = torch.randint(0, V, (B, W * ps), generator=g, dtype=torch.int32).cuda()
    rules = binding.LogitRules(history=history, history_len=prefix, prompt_len=prompt, repetition=torch.full((B,), 1.2, device="cuda"),
                               frequency=torch.full((B,), 0.1, device="cuda"))
    new = {k: torch.empty(s, dtype=dt, device="cuda") for k, s in (
        ("q", (layers, B, N, heads, D)), ("keys", (layers, B * N, kv, D)), ("values", (layers, B * N, kv, D)), ("target", (B, N, V)), ("draft", (B, n_int, V)))}
    u_draw, u_test = torch.empty((B, N), device="cuda"), torch.empty((B, N, 2), device="cuda")
    target, draft, cand = torch.empty_like(new["target"]), torch.empty_like(new["draft"]), torch.empty((B, N), **i32)
    att = [binding.TreeAttention(B, parent, heads, dt, cache.layer(0), W) for _ in range(layers)]
    caches = [cache.layer(l) for l in range(layers)]
    ver = binding.Verifier(B, parent, V, dt)
    tree_slots = torch.empty(B * N, dtype=torch.int64, device="cuda")
    back = [torch.empty((B * N, kv, D), device="cuda") for _ in range(2)]
    levels = [(0, 1), (1, 4), (4, 10)]

    def step():
        plan.mcsd_build_page_tables(prefix, N, slots=tree_slots)
        for l in range(layers):
            binding.mcsd_append_kv(caches[l], new["keys"][l], new["values"][l], tree_slots)
            att[l].mcsd_tree_attention(new["q"][l], caches[l], plan.table, prefix)
        target.copy_(new["target"]), draft.copy_(new["draft"])
        cand.fill_(-1)
        for lo, hi in levels:
            binding.mcsd_apply_logit_rules(draft, parent, cand, rules, node_begin=lo, node_end=hi)
            binding.mcsd_sample_candidates(draft, parent, u_draw, 1.0, 1, node_begin=lo, node_end=hi, cand=cand)
        binding.mcsd_apply_logit_rules(target, parent, cand, rules)
        out = ver.mcsd_verify(target, draft, cand, u_test, 1.0, 1)
        binding.mcsd_gather_accepted_pages(cache, plan.table, prefix, out.path_nodes, out.accept_len)
        binding.mcsd_read_kv(caches[1], tree_slots, keys=back[0], values=back[1])
        at = prefix[:, None].long() + torch.arange(gamma + 1, device="cuda")
        history.scatter_(1, at, torch.where(out.tokens >= 0, out.tokens, history.gather(1, at)))
        prefix.add_(out.accept_len + 1)

    def fresh():
        for k in ("q", "keys", "values"):
            new[k].copy_(torch.randn(new[k].shape, generator=g))
        new["target"].copy_(2 * torch.randn((B, N, V), generator=g))
        new["draft"].copy_(new["target"][:, :n_int].float() + 0.5 * torch.randn((B, n_int, V), generator=g).cuda())
        for u in (u_draw, u_test):
            u.copy_(torch.rand(u.shape, generator=g).clamp(1e-3, 1 - 1e-3))

    assert n_int == 10 and int(binding.load_library().mcsd_tree_depth(parent.ctypes.data, N)) == gamma
    state = (cache.pages, plan.table, plan.held, plan.ring, plan.ring_state, prefix, history)
    kept = [t.clone() for t in state]
    fresh()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):                    # warm-up, as graph capture asks for
        step()
    torch.cuda.current_stream().wait_stream(side)
    for t, k in zip(state, kept):
        t.copy_(k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    moved = 0
    for _ in range(5):
        fresh()
        pages, table, held, ring, (head, free, _, _), start, past = (t.cpu().numpy().copy() for t in state)
        graph.replay()
        torch.cuda.synchronize()
        want = ref.page_tables(start, np.full(B, N), table, held, ring, int(head), int(free), ps)
        assert np.array_equal(plan.table.cpu().numpy(), want[0]) and np.array_equal(plan.held.cpu().numpy(), want[1])
        assert plan.ring_state.tolist() == [want[3], want[4], 0, 0] and np.array_equal(tree_slots.cpu().numpy(), want[5]) and (want[7] == 0).all()
        f = lambda t: t.float().cpu().numpy()
        stored = np.stack([ref.append(pages[l], f(new["keys"][l]), f(new["values"][l]), want[5], D, ps) for l in range(layers)])
        for l in range(layers):
            o, lse, tol, tol_lse = ref.attention(f(new["q"][l]), stored[l], want[0], start, parent, D, ps, D ** -0.5, torch.finfo(dt).eps)
            assert (np.abs(f(att[l].out) - o) <= tol).all() and (np.abs(f(att[l].lse) - lse) <= tol_lse).all()
        kw = dict(history=past, history_len=start, prompt_len=np.array(lengths), repetition=np.full(B, np.float32(1.2)), frequency=np.full(B, np.float32(0.1)))
        for got, raw in ((target, new["target"]), (draft, new["draft"])):
            w, size, _ = ref.logit_rules(f(raw), parent, cand.cpu().numpy(), **kw)
            assert (np.abs(f(got) - w) <= torch.finfo(dt).eps / 2 * np.abs(w) + 2.0 ** -22 * size).all()
        # the sampler and the verification on the same inputs outside of the graph
        again = torch.full((B, N), -1, **i32)
        for lo, hi in levels:
            binding.mcsd_sample_candidates(draft, parent, u_draw, 1.0, 1, node_begin=lo, node_end=hi, cand=again)
        assert torch.equal(again, cand)
        accept, path, tokens = (t.clone() for t in (ver.accept_len, ver.path_nodes, ver.tokens))
        out = ver.mcsd_verify(target, draft, cand, u_test, 1.0, 1)
        assert torch.equal(out.accept_len, accept) and torch.equal(out.path_nodes, path) and torch.equal(out.tokens, tokens)
        rows = ref.move(stored, want[0], start, path.cpu().numpy(), accept.cpu().numpy(), D, ps)
        assert np.array_equal(cache.pages.cpu().numpy(), rows)
        for i, slot in enumerate(want[5]):
            for b_, w in zip(back, ref.row_values(rows[1], int(slot) // ps, int(slot) % ps, D, ps)):
                assert np.array_equal(f(b_[i]), w.astype(np.float32))
        assert prefix.tolist() == [int(s) + int(a) + 1 for s, a in zip(start, accept)]
        for b in range(B):
            n = int(accept[b]) + 1
            past[b, start[b]:start[b] + n] = tokens[b, :n].cpu().numpy()
        assert np.array_equal(history.cpu().numpy(), past)
        moved += int((accept > 0).sum())
    assert moved > 0


def test_new_buffers_are_ready_for_any_stream():
    """Objects made while their stream is busy, used on another stream at once: nothing that was enqueued for making them
    comes after the call."""
    parent = synth.tree_from_kconfig([2])
    B, N, ps, D, heads = 2, 3, 16, 64, 2
    g = torch.Generator().manual_seed(13)
    rows = torch.randn((2 * ps * B, heads, D), generator=g).cuda()
    q = torch.randn((B, N, heads, D), generator=g).to(torch.bfloat16).cuda()
    lengths, start = torch.full((B,), 20, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    slots, tree_slots = (torch.empty(n, dtype=torch.int64, device="cuda") for n in (20 * B, N * B))

    def use(make, stream):
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            made = []
            for f in make:                           # (each made on the busy stream, used on this one)
                with torch.cuda.stream(torch.cuda.default_stream()):
                    if stream != torch.cuda.default_stream():
                        torch.cuda._sleep(20_000_000)        # about 10 ms
                    made.append(f(*made))
                if len(made) == 1:
                    made[0].mcsd_build_page_tables(start, 20, slots=slots)
                    made[0].mcsd_build_page_tables(lengths, N, slots=tree_slots)
                elif len(made) == 2:
                    binding.mcsd_append_kv(made[1], rows[:20 * B], rows[:20 * B].flip(0), slots)
                    binding.mcsd_append_kv(made[1], rows[-N * B:], rows[:N * B], tree_slots)
                else:
                    r = made[2].mcsd_tree_attention(q, made[1], made[0].table, lengths)
        torch.cuda.synchronize()
        return r.out, r.lse, made[1].pages, made[0].table, made[0].ring_state

    make = [lambda: binding.PageTables.empty(B, 4, 9, ps), lambda p: binding.KvCache.empty(9, heads, D, ps),
            lambda p, c: binding.TreeAttention(B, parent, heads, q.dtype, c, 4)]
    want = use(make, torch.cuda.default_stream())
    got = use(make, torch.cuda.Stream())
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and (want[0] != 0).any()
