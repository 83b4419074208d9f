"""The bounded wait of the node kernel's exchange really gives up, and the kernel still returns.

Nothing here hangs or faults a GPU: the exchange barrier of a single-CTA cluster is armed for
16 bytes more than are sent (MCSD_OPT_TEST_EXTRA_TX), so the wait of the CTA's leader warp is a
wait for a flag nothing sets; with a budget of a few polls (MCSD_OPT_WAIT_POLLS) it runs out
within microseconds.  The kernel then stops waiting, arming and sending, finishes its items
without results, meets the final cluster barrier and exits; the status words say TIMEOUT.  A
normal call right after it works again."""
import numpy as np
import pytest
import torch

from paper_2401_06706_b200 import binding, synth
from gpu_util import Guards, assert_parity, library_options, to_np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("entry", ["mcsd_verify", "mcsd_verify_path"])
def test_expired_exchange_wait_sets_timeout_and_returns(entry):
    assert torch.cuda.is_available(), "this test needs a CUDA device"
    w = synth.Workload("timeout", 3, 2000, "2", "fp32", "normal", 2.5, 1.0, 1.0, 1.0, 0, 606)
    inp = synth.make_inputs(w, "cuda")
    v = binding.Verifier(w.batch, inp.parent, w.vocab, torch.float32, "cuda")
    guards = Guards(v)
    with library_options(cluster=1, wait_polls=4, test_extra_tx=16, pdl=0):
        out = getattr(v, entry)(inp.target, inp.draft, inp.cand, inp.unif, 1.0, 0)
        guards.check()                       # synchronises: the kernel has returned
    st = to_np(out.status)
    assert (st & binding.STATUS_TIMEOUT).all(), st
    # the library and the context are as usable as before
    out = getattr(v, entry)(inp.target, inp.draft, inp.cand, inp.unif, 1.0, 0)
    guards.check()
    assert not (to_np(out.status) & binding.STATUS_TIMEOUT).any()
    assert_parity(inp, out, sequential=(entry == "mcsd_verify_path"))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("prefixes", [[40, -1, 3], [1500, -1, 700]])
def test_expired_waits_of_the_attention_of_many_rows_give_nan_rows_and_return(D, prefixes):
    """The same for the kernel of tree attention whose roles wait for one another: a barrier expects an arrival that never
    comes, the waits run out, all roles go on to their end, and every row of a used entry is NaN (of items in one piece and of
    divided ones)."""
    g = torch.Generator().manual_seed(D)
    parent = synth.tree_from_kconfig([4, 4, 2, 2, 1])            # 181 rows per key head
    N, ps, longest = len(parent), 16, max(prefixes)
    W = -(-(longest + N) // ps)
    cache = binding.KvCache.empty(3 * W, 2, D, ps)
    rows = torch.randn((3 * W * ps, 2, D), generator=g).cuda()
    binding.mcsd_append_kv(cache, rows, rows.flip(0).contiguous(), torch.arange(3 * W * ps, device="cuda"))
    table = torch.arange(3 * W, dtype=torch.int32, device="cuda").view(3, W)
    prefix = torch.tensor(prefixes, dtype=torch.int32, device="cuda")
    q = torch.randn((3, N, 2, D), generator=g).to(torch.bfloat16).cuda()
    att = binding.TreeAttention(3, parent, 2, q.dtype, cache, W)
    right = att.mcsd_tree_attention(q, cache, table, prefix)
    out, lse = right.out.clone(), right.lse.clone()
    torch.cuda.synchronize()
    att.out.fill_(2.0)
    att.lse.fill_(3.0)
    with library_options(wait_polls=4, test_extra_tx=16):
        att.mcsd_tree_attention(q, cache, table, prefix)
        torch.cuda.synchronize()                                 # (it returned)
    used = prefix >= 0
    assert torch.isnan(att.out[used]).all() and torch.isnan(att.lse[used]).all()
    assert (att.out[~used] == 2).all() and (att.lse[~used] == 3).all()
    # the library and the context are as usable as before
    att.mcsd_tree_attention(q, cache, table, prefix)
    torch.cuda.synchronize()
    assert torch.equal(att.out[used], out[used]) and torch.equal(att.lse[used], lse[used])
