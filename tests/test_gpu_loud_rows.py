"""Attention of rows whose scores are so large that a float32 step of theirs is more than the range of an exponent: their weights are those of the largest
scores as the kernel has them, and finite, whichever kernel has the rows."""
import pytest
import torch

import test_gpu_ops_attention as trees
from paper_2401_06706_b200 import binding
from prompts_util import attend, check_attention, problem

pytestmark = pytest.mark.gpu
POWERS = [20, 24, 26, 28, 30, 34, 40, 70, 100]


def _in_reach(out, cache):
    """Rows are averages of cached values, which are within the largest of them (and a rounding)."""
    slots = torch.arange(cache.n_pages * cache.page_size, device="cuda")
    most = binding.mcsd_read_kv(cache, slots)[1].abs().max()
    assert torch.isfinite(out).all() and float(out.abs().max()) <= 1.01 * float(most)


@pytest.mark.parametrize("power", POWERS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("counts,heads,kv", [([1, 1], 4, 2), ([3, 2], 8, 2), ([9, 2], 2, 1), ([90, 70], 8, 2), ([300, 1], 2, 2)])
def test_chunks(power, D, counts, heads, kv):
    p = problem(44, [700, 301], counts, heads, kv, D, 16, torch.bfloat16)
    p.q[::3, 1] *= 2.0 ** power
    r = attend(p)
    check_attention(p, r)                            # (the tolerance of the loud rows is as large as their scores' steps)
    _in_reach(r.out, p.cache)

@pytest.mark.parametrize("power", POWERS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kconfig,heads,kv", [("", 4, 2), ("4x2x2x1", 2, 2), ("4x2x2x1", 4, 2), ("4x4x2x2x1", 4, 2), ("8x8x6", 2, 1)])
def test_trees(power, D, kconfig, heads, kv):
    parent, q, cache, table, prefix = trees._problem(45, 2, kconfig, heads, kv, D, 16, [700, 301], torch.bfloat16)
    q[:, ::3, 1] *= 2.0 ** power
    r = trees._run(q, cache, table, prefix, parent)
    trees._check(q, cache, table, prefix, parent, r.out, r.lse)
    _in_reach(r.out, cache)
