"""GPU parity of accumulated attention weights and of eviction by them against 64-bit statements of them on the same seeded inputs.

Tolerances, from the arithmetic: logits are sums of D exact products in fp32, so |dz| <= D 2^-23 scale sum|q_i k_i|
<= 128 * 1.2e-7 * 0.09 * 110 ~ 1.5e-4 at D = 128 and N(0,1) inputs.  A weight is off by at most 2 |dz| of itself
(its own logit and the denominator's): 3e-4 relative.  An output is a mean of values below 4.6 under such weights:
1.4e-3 absolute (the bar of the other attention tests, 2e-3, holds it); lse is off by |dz|.  bf16 results add half a
step, 2^-8 of the value.  Errors of independent roundings add as squares, so what is seen is two orders below."""
import numpy as np
import pytest
import torch

from paper_2609_20734_b200 import binding, synth
from tests import gpu_helpers as gh
from tests.cache_ops_ref import evict_reference, full_reference
from tests.helpers import make_problem

pytestmark = pytest.mark.gpu

RTOL_W = 3e-4
ONES = dict(dtype=torch.uint8, device="cuda")


def rows_close(out, lse, ref, rlse, layers, requests, what=""):
    bf16 = out.dtype == torch.bfloat16
    o, e = out.float().cpu().numpy(), lse.cpu().numpy()
    for l in layers:
        for b in requests:
            tol = gh.ATOL_OUT + (np.abs(ref[l, b]) / 256 if bf16 else 0)
            assert np.isfinite(o[l, b]).all(), f"{what}: non-finite out at layer {l} request {b}"
            assert (np.abs(o[l, b] - ref[l, b]) <= tol).all(), f"{what}: out at layer {l} request {b}: {np.abs(o[l, b] - ref[l, b]).max()}"
            gh.assert_close(e[l, b], rlse[l, b], gh.ATOL_LSE, f"{what}: lse at layer {l} request {b}")


def new_weights(prob, slices=None, seed=1, max_batch=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = prob["table"].shape[1] * 16
    return torch.rand((slices or prob["kv_layers"], max_batch or prob["B"], prob["Hkv"], n), generator=g, device="cuda")


def weights_close(got, before, wts, prob, flags, gated, kv_index=None, what=""):
    """got == before + the sum of every recalled layer's weights, on flagged requests and positions < t only."""
    want = before.double().cpu().numpy()
    add = np.zeros_like(want)
    for (l, b, g), w in wts.items():
        if gated[l] and flags[b]:
            add[l if kv_index is None else kv_index[l], b, g, :len(w)] += w
    got = got.double().cpu().numpy()
    same = add == 0
    assert (got[same] == want[same]).all(), f"{what}: weights of other positions changed"
    err = np.abs(got - want - add)
    # the sum is rounded to fp32 once per layer: 2^-24 of values below 1 + group
    tol = RTOL_W * add + 1e-6
    assert (err <= tol).all(), f"{what}: {err.max()} at {np.unravel_index((err - tol).argmax(), err.shape)}"


# ------------------------------------------------------------------------------------------------ weighted
@pytest.mark.parametrize("D,Hq,Hkv", [(128, 8, 2), (128, 8, 1), (64, 4, 4), (64, 16, 8), (128, 2, 1)])
@pytest.mark.parametrize("layout,dtype", [("hnd", 0), ("nhd", 1)])
def test_weighted_parity_ragged(D, Hq, Hkv, layout, dtype):
    seq = [1, 15, 16, 17, 300, 999, 0]
    L, gated, flags = 3, [1, 0, 1], [1, 1, 0, 1, 1, 1, 0]
    prob = make_problem(500 + D + Hq, L, len(seq), Hq, Hkv, D, seq, layout=layout)
    ctx = gh.make_ctx(prob, [64, 32, 16], [4, 0, 1], gated, out_dtype=dtype)
    dev = gh.upload(prob)
    out, lse = gh.new_out(prob, fill=-3.0, dtype=torch.bfloat16 if dtype else torch.float32)
    w = new_weights(prob)
    before = w.clone()
    f = torch.tensor(flags, **ONES)
    ctx.full_decode_weighted(0, L, len(seq), dev["q"], dev["k"], dev["v"], dev["table"], dev["seq_lens"], f, w, out, lse)
    torch.cuda.synchronize()
    assert ctx.read_device_status() == 0
    ref, rlse, wts = full_reference(prob)
    take = [b for b in range(len(seq)) if flags[b]]
    rows_close(out, lse, ref, rlse, [0, 2], take, "weighted")
    weights_close(w, before, wts, prob, flags, gated, what="weighted")
    rest = torch.ones((L, len(seq)), dtype=torch.bool)
    for b in take:
        rest[[0, 2], b] = False
    assert (out.cpu()[rest] == -3.0).all() and (lse.cpu()[rest] == -3.0).all()


def test_weighted_lone_heads_long_history_and_scale():
    """One request whose units are cut into many spans, G = 8 and G = 1, and a logit scale of its own."""
    for Hq, Hkv, D in ((8, 1, 128), (1, 1, 64)):
        prob = make_problem(31 + Hq, 1, 1, Hq, Hkv, D, [20011])
        ctx = gh.make_ctx(prob, [64], [4], [1], sm_scale=0.3)
        dev = gh.upload(prob)
        out, lse = gh.new_out(prob)
        w = new_weights(prob)
        before = w.clone()
        ctx.full_decode_weighted(0, 1, 1, dev["q"], dev["k"], dev["v"], dev["table"], dev["seq_lens"],
                                 torch.ones(1, **ONES), w, out, lse)
        ref, rlse, wts = full_reference(prob, sm_scale=0.3)
        # logits are 0.3 / 0.088 times larger: so are their errors
        o = out.cpu().numpy()
        assert np.abs(o - ref).max() <= 4 * gh.ATOL_OUT and np.abs(lse.cpu().numpy() - rlse).max() <= 4 * gh.ATOL_LSE
        add = w.double().cpu().numpy() - before.double().cpu().numpy()
        want = np.zeros_like(add)
        for (l, b, g), x in wts.items():
            want[l, b, g, :len(x)] = x
        assert (np.abs(add - want) <= 4 * RTOL_W * want + 1e-6).all()


def test_weighted_layers_that_share_a_slice_and_little_scratch():
    """Layers on one cache slice add to the same values; a scratch of one layer, of two, of all give the same bits."""
    seq = [130, 700]
    kv_index, gated, flags = [1, 0, 1, 1, 0], [1, 1, 0, 1, 1], [1, 1]
    prob = make_problem(77, 5, 2, 8, 2, 128, seq, kv_layers=2)
    ctx = gh.make_ctx(prob, [64] * 5, [4] * 5, gated, kv_index=kv_index, max_batch=3)
    dev = gh.upload(prob)
    ref, rlse, wts = full_reference(prob, kv_index)
    got = []
    for layers in (1, 2, 5):
        out, lse = gh.new_out(prob, fill=0.0)
        w = new_weights(prob, slices=2, max_batch=3)
        before = w.clone()
        ctx.full_decode_weighted(0, 5, 2, dev["q"], dev["k"], dev["v"], dev["table"], dev["seq_lens"],
                                 torch.ones(2, **ONES), w, out, lse, scratch=ctx.full_decode_weighted_scratch(layers))
        rows_close(out, lse, ref, rlse, [0, 1, 3, 4], [0, 1], f"{layers} layers at a time")
        weights_close(w, before, wts, prob, flags, gated, kv_index, f"{layers} layers at a time")
        got.append(w)
    assert all((x - got[0]).abs().max() <= 1e-5 for x in got)
    # only layers [1, 4) of the stack
    w = torch.zeros_like(got[0])
    out, lse = gh.new_out(prob, fill=9.0)
    ctx.full_decode_weighted(1, 4, 2, dev["q"], dev["k"], dev["v"], dev["table"], dev["seq_lens"], torch.ones(2, **ONES), w, out, lse)
    assert (out[[0, 2, 4]] == 9.0).all()
    weights_close(w, torch.zeros_like(w), {k: x for k, x in wts.items() if 1 <= k[0] < 4}, prob, flags, gated, kv_index, "layers 1-3")


def test_weighted_poisoned_tail_without_lse_graph_and_repeat():
    """NaN in slots past t - 1 and -1 in table entries past the last page are never used; lse may be absent; a captured
    call replays to the same bits as the eager one and reads lengths and flags on the device."""
    seq = [37, 130, 1]
    prob = make_problem(9, 2, 3, 4, 1, 128, seq)
    ref, rlse, wts = full_reference(prob)
    lay = prob["layout"]
    for b, t in enumerate(seq):
        blk = int(prob["table"][b, (t - 1) // 16])
        for l in range(2):
            for slot in range(t % 16, 16) if t % 16 else []:
                off = l * lay.layer_stride + blk * lay.block_stride + slot * lay.token_stride
                prob["k"][off:off + 128] = 0x7FC0
                prob["v"][off:off + 128] = 0x7FC0
    ctx = gh.make_ctx(prob, [48] * 2, [4] * 2, [1] * 2)
    dev = gh.upload(prob)
    f = torch.ones(3, **ONES)
    scratch = ctx.full_decode_weighted_scratch()
    scratch.fill_(0xFF)  # NaN: nothing of it is read before it is written

    def call(w, out, lse):
        ctx.full_decode_weighted(0, 2, 3, dev["q"], dev["k"], dev["v"], dev["table"], dev["seq_lens"], f, w, out, lse, scratch=scratch)

    w, (out, lse) = new_weights(prob), gh.new_out(prob, fill=0.0)
    before = w.clone()
    call(w, out, lse)
    rows_close(out, lse, ref, rlse, [0, 1], [0, 1, 2], "poisoned")
    weights_close(w, before, wts, prob, [1, 1, 1], [1, 1], what="poisoned")
    w2, (out2, _) = before.clone(), gh.new_out(prob, fill=0.0)
    call(w2, out2, None)
    assert torch.equal(w, w2) and torch.equal(out, out2)
    w3, (out3, lse3) = before.clone(), gh.new_out(prob, fill=0.0)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(w3, out3, lse3)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(w, w3) and torch.equal(out, out3) and torch.equal(lse, lse3)
    dev["seq_lens"].copy_(torch.tensor([20, 130, 1]))
    f.copy_(torch.tensor([1, 0, 0]))
    w3.copy_(before)
    g.replay()
    short = dict(prob, seq_lens=np.array([20, 130, 1], np.int32))
    _, _, wts = full_reference(short)
    weights_close(w3, before, wts, short, [1, 0, 0], [1, 1], what="replayed with other lengths")


# ------------------------------------------------------------------------------------------------ eviction
def weight_pattern(name, shape, rng):
    if name == "ties":
        return rng.integers(0, 4, shape).astype(np.float32)
    if name == "zeros":
        return np.zeros(shape, np.float32)
    if name == "odd":  # signed zeros, negatives, infinities, denormals, NaN
        pool = np.array([0.0, -0.0, -1.5, 2.0, np.inf, -np.inf, 1e-42, -1e-42, np.nan, 3.0, 1e30], np.float32)
        return pool[rng.integers(0, len(pool), shape)]
    if name == "rising":
        return np.broadcast_to(np.arange(shape[-1], dtype=np.float32), shape).copy()
    return np.exp(2 * rng.standard_normal(shape)).astype(np.float32)


def run_evict(prob, w_host, budget, sinks, recent, mask=None, with_kept=True, max_batch=None, kv_index=None):
    L, B = prob["L"], prob["B"]
    ctx = gh.make_ctx(prob, [16] * L, [0] * L, [1] * L, max_batch=max_batch, kv_index=kv_index)
    dev = gh.upload(prob)
    w = torch.full((w_host.shape[0], max_batch or B, *w_host.shape[2:]), 5.0, device="cuda")
    w[:, :B] = torch.from_numpy(w_host).cuda()
    kept = torch.full((w_host.shape[0], B, prob["Hkv"], budget), -7, dtype=torch.int32, device="cuda") if with_kept else None
    m = None if mask is None else torch.tensor(mask, **ONES)
    ctx.evict(B, w, dev["k"], dev["v"], dev["table"], dev["seq_lens"], budget, sinks, recent, mask=m, kept=kept)
    torch.cuda.synchronize()
    assert max_batch is None or (w[:, B:] == 5.0).all()
    bits = [dev[c].view(torch.int16).cpu().numpy().view(np.uint16) for c in ("k", "v")]
    return ctx, bits[0], bits[1], w[:, :B].cpu().numpy(), dev["seq_lens"].cpu().numpy(), None if kept is None else kept.cpu().numpy()


def check_evict(prob, w_host, budget, sinks, recent, **kw):
    want = evict_reference(prob, w_host, budget, sinks, recent, kw.get("mask"))
    ctx, *got = run_evict(prob, w_host, budget, sinks, recent, **kw)
    for name, a, b in zip(("k", "v", "weights", "seq_lens", "kept"), got, want):
        if a is not None:
            np.testing.assert_array_equal(a, b, err_msg=name)
    return ctx


@pytest.mark.parametrize("pattern", ["random", "ties", "zeros", "odd", "rising"])
@pytest.mark.parametrize("budget,sinks,recent", [(100, 4, 32), (16, 0, 0), (33, 0, 33), (7, 7, 0), (1, 0, 1), (1, 0, 0), (257, 17, 100)])
def test_evict_patterns_and_budgets(pattern, budget, sinks, recent):
    seq = [1, 16, 257, 258, 700, 1500]
    prob = make_problem(11, 2, len(seq), 4, 2, 64, seq, layout="hnd")
    w = weight_pattern(pattern, (2, len(seq), 2, prob["table"].shape[1] * 16), np.random.default_rng(budget))
    ctx = check_evict(prob, w, budget, sinks, recent)
    assert ctx.read_device_status() == 0


@pytest.mark.parametrize("D,Hkv,layout", [(128, 1, "nhd"), (128, 3, "hnd"), (64, 5, "nhd")])
def test_evict_layouts_masks_slices(D, Hkv, layout):
    seq = [900, 31, 5000, 1025, 640]
    prob = make_problem(12, 3, len(seq), Hkv, Hkv, D, seq, layout=layout, kv_layers=2)
    w = weight_pattern("random", (2, len(seq), Hkv, prob["table"].shape[1] * 16), np.random.default_rng(3))
    check_evict(prob, w, 640, 4, 128, mask=[1, 1, 1, 0, 1], max_batch=7, kv_index=[0, 1, 0])
    check_evict(prob, w, 1024, 0, 1, with_kept=False, kv_index=[0, 1, 0])


@pytest.mark.parametrize("t,budget", [(2053, 2052), (4097, 4096), (9000, 8999), (30000, 17), (70000, 33333), (300001, 100000)])
def test_evict_lengths(t, budget):
    """One position too many, and long histories (few units: one unit is worked on by several CTAs)."""
    prob = make_problem(13, 1, 1, 2, 1, 128, [t])
    w = weight_pattern("random", (1, 1, 1, prob["table"].shape[1] * 16), np.random.default_rng(t))
    check_evict(prob, w, budget, 4, min(12, budget - 4))


def test_evict_leaves_bad_lengths_and_says_so():
    prob = make_problem(14, 1, 3, 2, 2, 64, [50, 0, 60])
    w = weight_pattern("random", (1, 3, 2, prob["table"].shape[1] * 16), np.random.default_rng(1))
    ctx = check_evict(prob, w, 20, 1, 4)
    assert ctx.read_device_status() == 1
    # again on the shortened requests: nothing left to drop
    prob2 = make_problem(14, 1, 3, 2, 2, 64, [20, 7, 20])
    assert check_evict(prob2, w[..., :prob2["table"].shape[1] * 16].copy(), 20, 1, 4).read_device_status() == 0


def test_weights_then_eviction_then_a_step():
    """As they are used: weights of two recalled passes, eviction to a budget, the next Full and Local pass.  After the
    eviction each slice and head holds its own kept positions: the references attend to exactly those."""
    seq, budget, sinks, recent = [600, 90, 333], 128, 4, 48
    prob = make_problem(21, 2, 3, 8, 2, 128, seq)
    ctx = gh.make_ctx(prob, [48] * 2, [4] * 2, [1] * 2)
    dev = gh.upload(prob)
    w = torch.zeros((2, 3, 2, prob["table"].shape[1] * 16), device="cuda")
    f = torch.ones(3, **ONES)
    out, lse = gh.new_out(prob)
    kept = torch.empty((2, 3, 2, budget), dtype=torch.int32, device="cuda")
    q2 = synth.gauss_bf16_tensor(99, synth.STREAM_Q, prob["q"].shape)
    q2_dev = synth.bf16_bits_to_torch(q2, "cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for q in (dev["q"], q2_dev):
            ctx.full_decode_weighted(0, 2, 3, q, dev["k"], dev["v"], dev["table"], dev["seq_lens"], f, w, out, lse)
        ctx.evict(3, w, dev["k"], dev["v"], dev["table"], dev["seq_lens"], budget, sinks, recent, kept=kept)
        ctx.full_decode_gated(0, 2, 3, q2_dev, dev["k"], dev["v"], dev["table"], dev["seq_lens"], f, out, lse)
    g.replay()
    torch.cuda.synchronize()
    assert dev["seq_lens"].tolist() == [128, 90, 128]
    _, _, w1 = full_reference(prob)
    _, _, w2 = full_reference(dict(prob, q=q2))
    wref = np.zeros(w.shape)
    for x in (w1, w2):
        for (l, b, h), a in x.items():
            wref[l, b, h, :len(a)] += a
    # the kept sets of the summed weights, except where two candidates are nearer than the weights' error
    got = kept.cpu().numpy()
    for l in range(2):
        for b, t in enumerate(seq):
            for h in range(2):
                k = got[l, b, h][got[l, b, h] >= 0]
                assert len(set(k)) == min(t, budget) and (np.diff(k) > 0).all()
                if t > budget:
                    gone = np.setdiff1d(np.arange(t), k)
                    assert gone.min() >= sinks and gone.max() < t - recent
                    stay = k[(k >= sinks) & (k < t - recent)]
                    assert wref[l, b, h, stay].min() >= wref[l, b, h, gone].max() * (1 - 2 * RTOL_W) - 2e-6
    after = dict(prob, q=q2, seq_lens=np.minimum(prob["seq_lens"], budget).astype(np.int32), k=prob["k"].copy(), v=prob["v"].copy())
    lay = prob["layout"]
    for l in range(2):
        for b, t in enumerate(after["seq_lens"]):
            for h in range(2):
                i, src = np.arange(t), got[l, b, h, :t].astype(np.int64)
                at = [(l * lay.layer_stride + prob["table"][b, x // 16].astype(np.int64) * lay.block_stride
                       + (x % 16) * lay.token_stride + h * lay.head_stride)[:, None] + np.arange(128) for x in (i, src)]
                after["k"][at[0]], after["v"][at[0]] = prob["k"][at[1]], prob["v"][at[1]]
    ref, rlse, _ = full_reference(after)
    rows_close(out, lse, ref, rlse, [0, 1], [0, 1, 2], "after the eviction")
    assert ctx.read_device_status() == 0


def test_weighted_more_units_than_a_grid_axis_holds():
    """128 requests x 513 heads of one position each: every weight is 1 and every output its value row."""
    B, H, D = 128, 513, 64
    prob = make_problem(41, 1, 1, H, H, D, [1])
    ctx = gh.make_ctx(dict(prob, table=np.zeros((B, 2), np.int32)), [16], [0], [1], max_batch=B)
    dev = gh.upload(prob)
    q = dev["q"].expand(1, B, H, D).contiguous()
    table = torch.full((B, 2), int(prob["table"][0, 0]), dtype=torch.int32, device="cuda")
    w = torch.zeros((1, B, H, 32), device="cuda")
    out = torch.zeros((1, B, H, D), device="cuda")
    ctx.full_decode_weighted(0, 1, B, q, dev["k"], dev["v"], table, torch.ones(B, dtype=torch.int32, device="cuda"),
                             torch.ones(B, **ONES), w, out)
    torch.cuda.synchronize()
    assert ctx.read_device_status() == 0
    # one term: e^(z - lse) is 1 up to the rounding of exp and of 1 / l, the value passes through parts of bf16 unchanged
    assert (w[..., 0] - 1).abs().max() <= 1e-6 and (w[..., 1:] == 0).all()
    lay = prob["layout"]
    rows = np.stack([prob["v"][int(prob["table"][0, 0]) * lay.block_stride + h * lay.head_stride:][:D] for h in range(H)])
    want = torch.from_numpy(synth.bf16_bits_to_f32(rows))
    assert (out[0].cpu() - want).abs().max() <= 1e-6 * want.abs().max()


def test_evict_on_a_side_stream_captured_and_replayed():
    """The call on a stream of its own equals the one on the default stream; a captured one reads lengths, weights and the
    mask on the device each time, and a second replay on shortened requests changes nothing."""
    seq, budget = [700, 90, 333], 128
    prob = make_problem(23, 2, 3, 2, 2, 64, seq)
    w_host = weight_pattern("random", (2, 3, 2, prob["table"].shape[1] * 16), np.random.default_rng(8))
    want = evict_reference(prob, w_host, budget, 4, 48, [1, 1, 0])
    ctx = gh.make_ctx(prob, [16] * 2, [0] * 2, [1] * 2)
    dev = gh.upload(prob)
    w = torch.from_numpy(w_host).cuda()
    m = torch.zeros(3, **ONES)
    kept = torch.full((2, 3, 2, budget), -7, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        ctx.evict(3, w, dev["k"], dev["v"], dev["table"], dev["seq_lens"], budget, 4, 48, mask=m, kept=kept)
    g.replay()  # nobody may be shortened yet
    torch.cuda.synchronize()
    assert dev["seq_lens"].tolist() == seq and (kept == -7).all()
    m.copy_(torch.tensor([1, 1, 0]))
    for _ in range(2):
        g.replay()
        torch.cuda.synchronize()
        got = [dev["k"].view(torch.int16).cpu().numpy().view(np.uint16), dev["v"].view(torch.int16).cpu().numpy().view(np.uint16),
               w.cpu().numpy(), dev["seq_lens"].cpu().numpy()]
        for name, a, b in zip(("k", "v", "weights", "seq_lens"), got, want):
            np.testing.assert_array_equal(a, b, err_msg=name)
    dev2, w2 = gh.upload(prob), torch.from_numpy(w_host).cuda()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        ctx.evict(3, w2, dev2["k"], dev2["v"], dev2["table"], dev2["seq_lens"], budget, 4, 48, mask=m)
    side.synchronize()
    assert torch.equal(w, w2) and torch.equal(dev["k"].view(torch.int16), dev2["k"].view(torch.int16)) and \
        torch.equal(dev["seq_lens"], dev2["seq_lens"])
    assert ctx.read_device_status() == 0


def test_weights_are_read_in_16_byte_pieces_or_refused():
    prob = make_problem(24, 1, 1, 2, 1, 64, [40])
    ctx = gh.make_ctx(prob, [16], [0], [1])
    dev = gh.upload(prob)
    n = prob["table"].shape[1] * 16
    off = torch.zeros(n + 1, device="cuda")[1:]
    with pytest.raises(binding.OdaError) as e:
        ctx.evict(1, off, dev["k"], dev["v"], dev["table"], dev["seq_lens"], 20)
    assert e.value.status == 1 and ctx.launch_count == 0
    # (the weighted pass takes any fp32 address)
    before = off.clone()
    out, lse = gh.new_out(prob)
    ctx.full_decode_weighted(0, 1, 1, dev["q"], dev["k"], dev["v"], dev["table"], dev["seq_lens"], torch.ones(1, **ONES), off, out, lse)
    _, _, wts = full_reference(prob)
    weights_close(off.view(1, 1, 1, n), before.view(1, 1, 1, n), wts, prob, [1], [1], what="odd address")
