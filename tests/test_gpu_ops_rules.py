"""mcsd_apply_logit_rules against a plain statement in 64 bits."""
import ctypes

import numpy as np
import pytest
import torch

import ops_reference as ref
from paper_2401_06706_b200 import binding, synth

pytestmark = pytest.mark.gpu
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _tree(kconfig):
    return synth.tree_from_kconfig(synth.parse_kconfig(kconfig))


def _inputs(B, kconfig, V, dtype, seed, *, history=50, bias=9, mask="table", device="cuda"):
    g = torch.Generator().manual_seed(seed)
    parent = _tree(kconfig)
    N = len(parent)
    ri = lambda lo, hi, shape: torch.randint(lo, hi, shape, generator=g, dtype=torch.int32)
    x = {"logits": (3 * torch.randn((B, N, V), generator=g)).to(dtype)}
    few = ri(0, V, (B, max(history // 4, 1)))
    x["history"] = torch.gather(few, 1, torch.randint(0, few.shape[1], (B, history), generator=g)) if history else ri(0, V, (B, 0))
    if history > 6:
        x["history"][:, 3] = -1                      # padding and foreign tokens are ignored
        x["history"][:, 5] = V
        x["history"][:, 6] = -2**31
    x["history_len"] = ri(0, history + 4, (B,))      # some longer than the row: clipped
    x["prompt_len"] = ri(0, history + 1, (B,))
    x["repetition"] = 1 + torch.rand((B,), generator=g)
    x["frequency"] = torch.rand((B,), generator=g) - 0.3
    x["presence"] = torch.rand((B,), generator=g)
    x["bias_ids"] = ri(-2, V + 2, (B, bias))
    if bias > 4:
        x["bias_ids"][:, 4] = x["bias_ids"][:, 1]    # an id twice: the later entry counts
    x["bias_values"] = 5 * torch.randn((B, bias), generator=g)
    cand = ri(0, V, (B, N))
    cand[:, N // 2:] = cand[:, :N - N // 2].clone()          # the same token again along a path
    if history:
        cand[:, ::3] = x["history"][:, :1]
    if N > 2:
        cand[0, 1] = -1
        cand[0, 2] = V + 7
    words = (V + 31) // 32
    if mask == "none":
        x["masks"] = x["mask_index"] = None
    else:
        n = 7 if mask == "table" else B * N
        x["masks"] = ri(-2**31, 2**31 - 1, (n, words))
        x["masks"][0] = 0                            # leaves nothing
        x["masks"][1] = -1                           # leaves everything
        x["mask_index"] = ri(-2, n, (B, N)) if mask == "table" else None
    x = {k: (None if v is None else v.to(device)) for k, v in x.items()}
    return parent, x, cand.to(device)


def _reference(parent, x, cand, nodes=None):
    f = lambda t: None if t is None else (t.float() if t.dtype in (torch.bfloat16, torch.float16) else t).cpu().numpy()
    kw = {k: f(v) for k, v in x.items() if k != "logits"}
    return ref.logit_rules(f(x["logits"]), parent, f(cand), nodes=nodes, **kw)


def _rules(x):
    return binding.LogitRules(**{k: v for k, v in x.items() if k != "logits"})


def _close(got, want, size, dtype):
    """One rounding to the type (half a step, of the smallest normal number at least) behind at most four in float32."""
    got = got.float().cpu().numpy().astype(np.float64)
    fi = torch.finfo(dtype)
    with np.errstate(invalid="ignore"):
        tol = fi.eps / 2 * np.maximum(np.abs(want), fi.tiny) + 4 * 2.0 ** -24 * size
        ok = (np.abs(got - want) <= tol) | (got == want) | (np.isnan(got) & np.isnan(want))
    over = np.isinf(got) & (np.abs(want) >= fi.max * (1 - fi.eps))
    assert (ok | over).all(), np.argwhere(~(ok | over))[:5]


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("B,kconfig,V,history,bias,mask", [
    (1, "", 1, 0, 0, "none"), (1, "2", 33, 5, 1, "rows"), (3, "4x2x2x1", 1000, 50, 9, "table"), (2, "1x1x1x1x1x1", 4099, 300, 40, "table"),
    (2, "2x2", 32000, 1500, 300, "table"), (1, "8x2x1", 65536, 40, 5, "rows"), (5, "3x3x1", 515, 2, 6, "none"), (2, "32", 8192, 7000, 1, "table")])
def test_rules_against_reference(dtype, B, kconfig, V, history, bias, mask):
    dt = DTYPES[dtype]
    parent, x, cand = _inputs(B, kconfig, V, dt, B * 1000 + V, history=history, bias=bias, mask=mask)
    want, size, _ = _reference(parent, x, cand)
    out = torch.full_like(x["logits"], 77.0)
    kept = x["logits"].clone()
    got = binding.mcsd_apply_logit_rules(x["logits"], parent, cand, _rules(x), out=out)
    _close(got, want, size, dt)
    assert torch.equal(x["logits"].view(torch.uint8), kept.view(torch.uint8))
    # in place: the same bits
    inplace = x["logits"].clone()
    binding.mcsd_apply_logit_rules(inplace, parent, cand, _rules(x))
    assert torch.equal(inplace.view(torch.uint8), got.view(torch.uint8))


@pytest.mark.parametrize("only", ["repetition", "frequency", "presence", "bias", "mask", "nothing"])
def test_single_rules(only):
    parent, x, cand = _inputs(3, "3x2", 2000, torch.bfloat16, 5, history=200, bias=20)
    groups = {"repetition": ["repetition"], "frequency": ["frequency"], "presence": ["presence"], "bias": ["bias_ids", "bias_values"],
              "mask": ["masks", "mask_index"], "nothing": []}
    for k in ("repetition", "frequency", "presence", "bias_ids", "bias_values", "masks", "mask_index"):
        if k not in groups[only]:
            x[k] = None
    want, size, _ = _reference(parent, x, cand)
    got = binding.mcsd_apply_logit_rules(x["logits"], parent, cand, _rules(x), out=torch.empty_like(x["logits"]))
    _close(got, want, size, torch.bfloat16)
    if only == "nothing":
        assert torch.equal(got.view(torch.uint8), x["logits"].view(torch.uint8))


@pytest.mark.parametrize("dtype", sorted(DTYPES))
def test_odd_strides_rows_in_range_and_padding_kept(dtype):
    """Rows at odd offsets (element loads), a node range, draft rows; what lies outside is left as it was."""
    dt = DTYPES[dtype]
    parent, x, cand = _inputs(2, "3x2x1", 701, dt, 9, history=90)
    n_int = int((np.bincount(parent[1:], minlength=len(parent)) > 0).sum())
    base = torch.full((2, n_int, 709), 5.0, dtype=dt, device="cuda")
    base[:, :, :701] = x["logits"][:, :n_int]
    view = base[:, :, :701]
    x["logits"] = view
    want, size, _ = _reference(parent, x, cand, nodes=range(1, 3))
    out_base = torch.full((2, n_int, 703), -3.0, dtype=dt, device="cuda")
    out = out_base[:, :, :701]
    binding.mcsd_apply_logit_rules(view, parent, cand, _rules(x), out=out, node_begin=1, node_end=3)
    _close(out[:, 1:3], want[:, 1:3], size[:, 1:3], dt)
    assert (out_base[:, :, 701:] == -3).all() and (out[:, 0] == -3).all() and (out[:, 3:] == -3).all()
    inplace = base.clone()
    binding.mcsd_apply_logit_rules(inplace[:, :, :701], parent, cand, _rules(x), node_begin=1, node_end=3)
    assert torch.equal(inplace[:, 1:3, :701], out[:, 1:3]) and (inplace[:, :, 701:] == 5).all()
    assert torch.equal(inplace[:, 0], base[:, 0]) and torch.equal(inplace[:, 3:], base[:, 3:])


def test_infinities_and_nan():
    """-inf, +inf and NaN logits go through the formula; a masked place is -inf whatever stood there."""
    parent, x, cand = _inputs(1, "2x2", 640, torch.float32, 3, history=600, bias=12, mask="table")
    g = torch.Generator().manual_seed(1)
    for value in (float("inf"), float("-inf"), float("nan"), torch.finfo(torch.float32).min, torch.finfo(torch.float32).max, 0.0, -0.0):
        at = torch.randint(0, 640, (40,), generator=g)
        x["logits"][:, :, at.cuda()] = value
    want, size, _ = _reference(parent, x, cand)
    got = binding.mcsd_apply_logit_rules(x["logits"], parent, cand, _rules(x), out=torch.empty_like(x["logits"]))
    with np.errstate(over="ignore"):
        want = np.where(np.abs(want) > np.finfo(np.float32).max, np.copysign(np.inf, want), want)
    _close(got, want, np.where(np.isfinite(size), size, 0), torch.float32)


def test_mask_rows_that_are_not_there():
    parent, x, cand = _inputs(3, "2", 100, torch.float16, 4, mask="table")
    x["mask_index"][1, 2] = 7
    want, size, status = _reference(parent, x, cand)
    got_status = torch.tensor([1, 0, 4], dtype=torch.int32, device="cuda")
    got = binding.mcsd_apply_logit_rules(x["logits"], parent, cand, _rules(x), out=torch.empty_like(x["logits"]), status=got_status)
    _close(got, want, size, torch.float16)
    assert list(status) == [0, 32, 0] and got_status.tolist() == [1, 32, 4]


def test_a_long_chain_counts_its_whole_path():
    """511 nodes below each other, all with the same few tokens."""
    parent = np.arange(-1, 511, dtype=np.int32)
    V = 600
    cand = torch.randint(0, 3, (1, 512), dtype=torch.int32, device="cuda") * 250
    x = {"logits": torch.randn((1, 512, V), device="cuda"), "frequency": torch.tensor([0.01], device="cuda"), "presence": torch.tensor([1.0], device="cuda"),
         "repetition": torch.tensor([1.5], device="cuda")}
    want, size, _ = ref.logit_rules(x["logits"].cpu().numpy(), parent, cand.cpu().numpy(), frequency=[np.float32(0.01)], presence=[1.0], repetition=[1.5])
    got = binding.mcsd_apply_logit_rules(x["logits"], parent, cand, _rules(x), out=torch.empty_like(x["logits"]))
    _close(got, want, size, torch.float32)


def test_a_mask_that_leaves_nothing_reaches_verify_as_no_mass():
    parent = _tree("2")
    t = torch.randn((1, 3, 50), device="cuda")
    d = torch.randn((1, 1, 50), device="cuda")
    cand = torch.tensor([[-1, 3, 4]], dtype=torch.int32, device="cuda")
    masks = torch.zeros((1, 2), dtype=torch.int32, device="cuda")
    rules = binding.LogitRules(masks=masks, mask_index=torch.zeros((1, 3), dtype=torch.int32, device="cuda"))
    binding.mcsd_apply_logit_rules(t, parent, None, rules)
    assert torch.isinf(t).all()
    out = binding.mcsd_verify(t, d, parent, cand, torch.full((1, 3, 2), 0.5, device="cuda"), 1.0, 0)
    assert int(out.status[0]) & binding.STATUS_NO_MASS and int(out.tokens[0, 0]) == -1


def test_capture_replay_with_changed_inputs_and_another_stream():
    parent, x, cand = _inputs(4, "2x2", 3000, torch.bfloat16, 8, history=100)
    rules, out = _rules(x), torch.empty_like(x["logits"])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        binding.mcsd_apply_logit_rules(x["logits"], parent, cand, rules, out=out)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        binding.mcsd_apply_logit_rules(x["logits"], parent, cand, rules, out=out)
    x["history_len"].fill_(60)
    x["logits"].neg_()
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    want, size, _ = _reference(parent, x, cand)
    _close(out, want, size, torch.bfloat16)


def test_empty_calls():
    parent, x, cand = _inputs(2, "2", 64, torch.float32, 1)
    before = x["logits"].clone()
    binding.mcsd_apply_logit_rules(x["logits"], parent, cand, _rules(x), node_begin=1, node_end=1)
    assert torch.equal(before, x["logits"]) and binding.mcsd_last_launch_count() == 0


@pytest.mark.parametrize("nodes,depth", [(448, 416), (447, 416), (448, 417), (512, 511)])
def test_the_deepest_trees_in_the_widest_slice(nodes, depth):
    """Shared memory of a call right at, below and above the default limit: 448 nodes, 416 levels and slices of 2048 tokens take
    48 KB of it beside the kernel's static part."""
    parent = np.concatenate([np.arange(-1, depth), np.full(nodes - depth - 1, depth - 1)]).astype(np.int32)   # a chain, the rest below its end
    assert len(parent) == nodes
    V, B, rows = 65536, 10, 3
    g = torch.Generator().manual_seed(nodes)
    x = {"logits": torch.randn((B, rows, V), generator=g).cuda(), "presence": torch.rand((B,), generator=g).cuda()}
    cand = torch.randint(0, V, (B, nodes), generator=g, dtype=torch.int32).cuda()
    cand[:, 2] = cand[:, 1]
    want, size, _ = _reference(parent, x, cand)
    got = binding.mcsd_apply_logit_rules(x["logits"], parent, cand, _rules(x), out=torch.empty_like(x["logits"]))
    _close(got, want, size, torch.float32)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("V", [701, 704])
@pytest.mark.parametrize("mask", [False, True])
def test_in_place_leaves_what_no_rule_concerns(dtype, V, mask):
    """Bit by bit, NaN payloads too, on rows that are read element by element (701) and by vectors with a ragged end."""
    dt = DTYPES[dtype]
    g = torch.Generator().manual_seed(V)
    bits = torch.int32 if dt == torch.float32 else torch.int16
    x = torch.randn((2, 3, V), generator=g).to(dt)
    nan = torch.tensor(0x7f812345, dtype=torch.int32).view(torch.float32) if dt == torch.float32 else torch.tensor({"bf16": 0x7f91, "fp16": 0x7d23}[dtype], dtype=torch.int16).view(dt)
    x.view(bits)[:, :, ::7] = nan.view(bits)
    x = x.cuda()
    ids = torch.tensor([[3, 700], [5, -1]], dtype=torch.int32, device="cuda")
    kw = dict(bias_ids=ids, bias_values=torch.ones((2, 2), device="cuda"))
    hidden = torch.zeros(V, dtype=torch.bool, device="cuda")
    if mask:
        hidden[[2, 64, 698]] = True
        words = torch.full(((V + 31) // 32,), -1, dtype=torch.int64)
        for i in (2, 64, 698):
            words[i // 32] -= 1 << (i % 32)          # (from all ones: the bit goes out)
        kw |= dict(masks=words.to(torch.int32)[None].cuda(), mask_index=torch.zeros((2, 3), dtype=torch.int32, device="cuda"))
    before = x.view(bits).clone()
    binding.mcsd_apply_logit_rules(x, _tree("2"), None, binding.LogitRules(**kw))
    touched = hidden.expand(2, V).clone()
    for b in range(2):
        touched[b, [int(i) for i in ids[b] if i >= 0]] = True
    same = x.view(bits) == before
    assert same[~touched[:, None].expand(2, 3, V)].all()
    assert torch.isneginf(x[:, :, hidden]).all() and (x[1, :, 5] == before.view(dt)[1, :, 5] + 1).all()


# ---------------------------------------------------------------- the slices of large batches
def _slice(B, V):
    """Tokens of one CTA: the widest slice of at most 2048 that gives every SM two CTAs."""
    sms, size = torch.cuda.get_device_properties(0).multi_processor_count, 2048
    while size > 512 and -(-V // size) * B < 2 * sms:
        size //= 2
    return size


def _device_reference(parent, x, cand, b):
    """(values, size of what was added up) of one sequence in 64 bits, [N, V], on the device."""
    V, N = x["logits"].shape[2], len(parent)
    ids, inside = x["history"][b].long(), (x["history"][b] >= 0) & (x["history"][b] < V)
    at = torch.arange(ids.numel(), device="cuda")
    inside &= at < x["history_len"][b].clamp(0, ids.numel())
    prompt = at < x["prompt_len"][b]
    base = torch.bincount(ids[inside & ~prompt], minlength=V).double()
    given = torch.bincount(ids[inside & prompt], minlength=V) > 0
    count = base.expand(N, V).clone()
    for n in range(N):
        for m in ref.path(parent, n)[:-1]:
            if 0 <= int(cand[b, m]) < V:
                count[n, int(cand[b, m])] += 1
    bias = torch.zeros(V, dtype=torch.float64, device="cuda")
    for i, v in zip(x["bias_ids"][b].tolist(), x["bias_values"][b].tolist()):
        if 0 <= i < V:
            bias[i] = v
    theta, f, p = (x[k][b].double() for k in ("repetition", "frequency", "presence"))
    l = x["logits"][b].double()
    pen = torch.where(l > 0, l / theta, l * theta)
    size = torch.maximum(l.abs(), pen.abs()) + f.abs() * count + p.abs() * (count > 0) + bias.abs()
    l = torch.where((count > 0) | given, pen, l) - f * count - p * (count > 0) + bias
    if x["masks"] is not None:
        token = torch.arange(V, device="cuda")
        for n in range(N):
            m = int(x["mask_index"][b, n])
            if 0 <= m < x["masks"].shape[0]:
                l[n, (x["masks"][m][token // 32] >> (token % 32)) & 1 == 0] = float("-inf")
    return l, size


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("B,kconfig,V,mask,slice_", [
    (64, "2x2x2x2", 50272, "table", 2048), (40, "4x2x2x1", 32003, "table", 2048), (20, "2x2x2x2", 32000, "none", 2048),
    (10, "4x2x2x1", 32000, "table", 1024), (12, "2x2x2x2", 32001, "table", 1024), (300, "3x3x1", 1100, "table", 2048)])
def test_slices_of_large_batches(dtype, B, kconfig, V, mask, slice_):
    """Slices of 1024 and 2048 tokens, the last one in part, several rows per warp; by vectors and by elements; both forms."""
    assert _slice(B, V) == slice_
    dt = DTYPES[dtype]
    parent, x, cand = _inputs(B, kconfig, V, dt, B + V, history=1000, bias=60, mask=mask)
    assert mask == "none" or len(x["mask_index"]) == B
    got = binding.mcsd_apply_logit_rules(x["logits"], parent, cand, _rules(x), out=torch.full_like(x["logits"], 77.0))
    inplace = x["logits"].clone()
    binding.mcsd_apply_logit_rules(inplace, parent, cand, _rules(x))
    assert torch.equal(inplace.view(torch.uint8), got.view(torch.uint8))
    fi, cpu_cand = torch.finfo(dt), cand.cpu()
    for b in range(0, B, max(B // 16, 1)):
        want, size = _device_reference(parent, x, cpu_cand, b)
        # one rounding to the type behind at most four in float32, as in _close
        tol = fi.eps / 2 * want.abs().clamp(min=fi.tiny) + 4 * 2.0 ** -24 * size
        assert (((got[b].double() - want).abs() <= tol) | (got[b].double() == want)).all()
