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
