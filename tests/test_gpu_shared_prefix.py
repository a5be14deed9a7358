"""GPU parity of the Full pass over shared prefixes against a 64-bit statement of it that shares nothing: every request's
whole history through its own table.  Tolerances as derived in test_gpu_cache_ops."""
import numpy as np
import pytest
import torch

from paper_2609_20734_b200 import synth
from tests import gpu_helpers as gh
from tests.cache_ops_ref import full_reference, share_prefixes
from tests.helpers import make_problem
from tests.test_gpu_cache_ops import ONES, rows_close

pytestmark = pytest.mark.gpu


def run_shared(prob, groups, prefix, flags, gated=None, dtype=0, fill=-3.0, ctx=None, dev=None, **kw):
    L, B = prob["L"], prob["B"]
    ctx = ctx or gh.make_ctx(prob, [64] * L, [4] * L, gated or [1] * L, out_dtype=dtype, **kw)
    dev = dev or gh.upload(prob)
    out, lse = gh.new_out(prob, fill=fill, dtype=torch.bfloat16 if dtype else torch.float32)
    scratch = ctx.full_decode_shared_scratch()
    scratch.fill_(0xFF)  # NaN: nothing of it is read before it is written
    gs = torch.tensor(groups, dtype=torch.int32, device="cuda")
    gp = torch.tensor(prefix, dtype=torch.int32, device="cuda")
    ctx.full_decode_shared(0, L, B, dev["q"], dev["k"], dev["v"], dev["table"], dev["seq_lens"], torch.tensor(flags, **ONES),
                           gs, gp, out, lse, scratch=scratch)
    torch.cuda.synchronize()
    return ctx, out, lse


def check_shared(prob, groups, prefix, flags=None, gated=None, dtype=0, status=0, kv_index=None, sm_scale=0.0):
    L, B = prob["L"], prob["B"]
    flags = flags or [1] * B
    gated = gated or [1] * L
    ctx, out, lse = run_shared(prob, groups, prefix, flags, gated, dtype, kv_index=kv_index, sm_scale=sm_scale)
    assert ctx.read_device_status() == status
    ref, rlse, _ = full_reference(prob, kv_index, sm_scale or None)
    take = [b for b in range(B) if flags[b] and prob["seq_lens"][b] > 0]
    layers = [l for l in range(L) if gated[l]]
    rows_close(out, lse, ref, rlse, layers, take, "shared")
    rest = torch.ones((L, B), dtype=torch.bool)
    for l in layers:
        rest[l, take] = False
    assert (out.cpu()[rest] == -3.0).all() and (lse.cpu()[rest] == -3.0).all()
    return out, lse


@pytest.mark.parametrize("D,Hq,Hkv", [(128, 8, 2), (128, 8, 1), (64, 4, 4), (64, 16, 8), (128, 2, 1)])
@pytest.mark.parametrize("layout,dtype", [("hnd", 0), ("nhd", 1)])
def test_shared_parity_groups(D, Hq, Hkv, layout, dtype):
    """Two groups with requests outside any group behind them, prefixes that end inside a page and inside a tile."""
    seq = [700, 612, 611, 999, 300, 310, 400, 5, 64]
    prob = make_problem(600 + D + Hq, 3, len(seq), Hq, Hkv, D, seq, layout=layout)
    share_prefixes(prob, [0, 4, 7], [611, 299], copy_pages=(2,))
    check_shared(prob, [0, 4, 7], [611, 299], flags=[1, 1, 0, 1, 1, 1, 1, 1, 0], gated=[1, 0, 1], dtype=dtype)


@pytest.mark.parametrize("prefix", [1, 15, 16, 17, 127, 128, 129, 144, 1024, 1300])
def test_shared_prefix_lengths(prefix):
    seq = [prefix + x for x in (1, 2, 16, 33, 200)]
    prob = make_problem(700 + prefix, 2, len(seq), 8, 2, 128, seq)
    share_prefixes(prob, [0, 5], [prefix])
    check_shared(prob, [0, 5], [prefix])


@pytest.mark.parametrize("B,G", [(2, 1), (17, 8), (33, 4), (40, 8), (128, 4), (128, 8), (65, 2)])
def test_shared_row_counts(B, G):
    """Query rows of a kv head below, at and above the matrix tile, in one and in several row blocks."""
    rng = np.random.default_rng(B)
    seq = [400 + int(x) for x in rng.integers(1, 60, B)]
    prob = make_problem(800 + B + G, 1, B, G, 1, 64, seq)
    share_prefixes(prob, [0, B], [400])
    check_shared(prob, [0, B], [400], dtype=G % 8 // 4)


def test_shared_prefix_reaches_the_end_of_a_request():
    """A prefix as long as the shortest request, and one that claims more than a request has."""
    seq = [320, 321, 500]
    prob = make_problem(41, 1, 3, 8, 2, 128, seq)
    share_prefixes(prob, [0, 3], [320])
    check_shared(prob, [0, 3], [320])
    check_shared(prob, [0, 3], [2000000000], flags=[1, 0, 0])
    prob = make_problem(42, 1, 3, 8, 2, 128, [320, 336, 500])  # the first request is shorter, and not flagged
    share_prefixes(prob, [1, 3], [336])
    check_shared(prob, [0, 3], [336], flags=[0, 1, 1])


def test_shared_nothing_to_share():
    """No groups, empty groups, groups of one, negative prefixes, nobody flagged."""
    seq = [100, 200, 300]
    prob = make_problem(43, 2, 3, 8, 2, 128, seq)
    check_shared(prob, [0], [])
    check_shared(prob, [0, 0, 1, 3, 3], [50, 50, -5, 70])
    check_shared(prob, [0, 3], [0])
    _, out, lse = run_shared(prob, [0, 3], [0], [0, 0, 0])
    assert (out == -3.0).all() and (lse == -3.0).all()


def test_shared_bad_groups_share_nothing_and_are_reported():
    seq = [100, 200, 300]
    prob = make_problem(44, 1, 3, 8, 2, 128, seq)
    for groups, prefix in (([0, 4], [64]), ([-1, 3], [64]), ([2, 0], [64]), ([0, 3, 1, 3], [0, 64, 64])):
        check_shared(prob, groups, prefix, status=8)


def test_shared_zero_length_request_is_reported_like_in_the_full_pass():
    prob = make_problem(45, 1, 4, 8, 2, 128, [200, 0, 210, 220])
    share_prefixes(prob, [0, 4], [130])
    check_shared(prob, [0, 4], [130], status=1)


def test_shared_poisoned_tails():
    """NaN in the slots past each request's last position, and in the pages nobody uses; -1 in unused table entries."""
    seq = [259, 270, 300]
    prob = make_problem(46, 1, 3, 8, 2, 128, seq)
    share_prefixes(prob, [0, 3], [250])
    lay = prob["layout"]
    used = np.zeros(prob["k"].size, bool)
    for b, t in enumerate(seq):
        j = np.arange(t)
        for g in range(2):
            at = (prob["table"][b, j // 16].astype(np.int64) * lay.block_stride + (j % 16) * lay.token_stride + g * lay.head_stride)
            used[(at[:, None] + np.arange(128)).reshape(-1)] = True
    prob["k"][~used] = 0x7FC0
    prob["v"][~used] = 0x7FC0
    check_shared(prob, [0, 3], [250])


def test_shared_layer_aliases_scale_and_layer_range():
    prob = make_problem(47, 4, 6, 8, 2, 128, [300 + i for i in range(6)], kv_layers=2)
    share_prefixes(prob, [0, 6], [288])
    check_shared(prob, [0, 6], [288], kv_index=[1, 0, 1, 0], sm_scale=0.2)
    ctx = gh.make_ctx(prob, [64] * 4, [4] * 4, [1, 0, 1, 1], kv_index=[1, 0, 1, 0])
    dev = gh.upload(prob)
    ref, rlse, _ = full_reference(prob, [1, 0, 1, 0])
    out, lse = gh.new_out(prob, fill=2.0)
    i32 = dict(dtype=torch.int32, device="cuda")
    ctx.full_decode_shared(1, 3, 6, dev["q"], dev["k"], dev["v"], dev["table"], dev["seq_lens"], torch.ones(6, **ONES),
                           torch.tensor([0, 6], **i32), torch.tensor([288], **i32), out, None)
    assert (out[[0, 1, 3]] == 2.0).all()
    rows_close(out, torch.from_numpy(rlse).float(), ref, rlse, [2], range(6), "layers 1-2")


def test_shared_many_spans_are_the_same_every_time_and_in_a_graph():
    """A prefix long enough that every unit is cut; eager, again, captured with other lengths, groups and flags."""
    seq = [9000 + 7 * i for i in range(6)]
    prob = make_problem(48, 2, 6, 8, 2, 128, seq)
    share_prefixes(prob, [0, 6], [8999])
    ctx = gh.make_ctx(prob, [64] * 2, [4] * 2, [1] * 2)
    dev = gh.upload(prob)
    _, out, lse = run_shared(prob, [0, 6], [8999], [1] * 6, ctx=ctx, dev=dev)
    ref, rlse, _ = full_reference(prob)
    rows_close(out, lse, ref, rlse, [0, 1], range(6), "long prefix")
    _, out2, lse2 = run_shared(prob, [0, 6], [8999], [1] * 6, ctx=ctx, dev=dev)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    i32 = dict(dtype=torch.int32, device="cuda")
    gs, gp, f = torch.tensor([0, 6], **i32), torch.tensor([8999], **i32), torch.ones(6, **ONES)
    out3, lse3 = gh.new_out(prob, fill=-3.0)
    scratch = ctx.full_decode_shared_scratch()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ctx.full_decode_shared(0, 2, 6, dev["q"], dev["k"], dev["v"], dev["table"], dev["seq_lens"], f, gs, gp, out3, lse3, scratch=scratch)
    g.replay()
    assert torch.equal(out, out3) and torch.equal(lse, lse3)
    short = np.array([8999, 4000, 8990, 8999, 130, 8999], np.int32)
    dev["seq_lens"].copy_(torch.from_numpy(short))
    gs.copy_(torch.tensor([0, 4]))
    gp.copy_(torch.tensor([3999]))
    f.copy_(torch.tensor([1, 1, 0, 1, 1, 0]))
    out3.fill_(-3.0)
    g.replay()
    ref, rlse, _ = full_reference(dict(prob, seq_lens=short))
    rows_close(out3, lse3, ref, rlse, [0, 1], [0, 1, 3, 4], "replayed with other lengths")
    assert (out3[:, [2, 5]] == -3.0).all()
    assert ctx.read_device_status() == 0


def test_shared_large_logits():
    """Logits of hundreds: the running maximum rises late in the prefix and only the last of it counts."""
    prob = make_problem(49, 1, 4, 8, 1, 128, [1500, 1510, 1520, 1530])
    share_prefixes(prob, [0, 4], [1490])
    k = synth.bf16_bits_to_f32(prob["k"])
    lay = prob["layout"]
    for j in range(1490):
        at = int(prob["table"][0, j // 16]) * lay.block_stride + (j % 16) * lay.token_stride
        k[at:at + 128] *= 0.01 + 6.0 * j / 1490
    prob["k"] = synth.f32_to_bf16_bits(k)
    share_prefixes(prob, [0, 4], [1490])
    ctx, out, lse = run_shared(prob, [0, 4], [1490], [1] * 4)
    ref, rlse, _ = full_reference(prob)
    # keys are six times longer: so are logits and their errors
    assert np.abs(out.cpu().numpy() - ref).max() <= 6 * gh.ATOL_OUT
    assert np.abs(lse.cpu().numpy() - rlse).max() <= 6 * gh.ATOL_LSE


@pytest.mark.parametrize("D,Hq,Hkv,B,dtype", [(128, 16, 8, 3, 1), (64, 16, 8, 3, 0), (64, 8, 8, 12, 1), (128, 64, 8, 17, 1), (64, 64, 8, 20, 0)])
def test_shared_long_runs_through_the_ring(D, Hq, Hkv, B, dtype):
    """Prefixes long enough, over enough heads and layers, that every CTA goes around its ring of tiles many times in one
    piece of work and through several pieces, with rows for one and for two row tiles."""
    L, prefix = (6, 3200) if B < 17 else (2, 3200)
    seq = [prefix + 1 + (5 * i) % 37 for i in range(B)]
    prob = make_problem(900 + D + B, L, B, Hq, Hkv, D, seq)
    share_prefixes(prob, [0, B], [prefix])
    ctx, out, lse = run_shared(prob, [0, B], [prefix], [1] * B, dtype=dtype)
    assert ctx.read_device_status() == 0
    # some requests, all heads and layers
    some = [0, 1, B - 1]
    few = dict(prob, B=len(some), q=prob["q"][:, some], table=prob["table"][some], seq_lens=prob["seq_lens"][some])
    ref, rlse, _ = full_reference(few)
    rows_close(out[:, some], lse[:, some], ref, rlse, range(L), range(len(some)), "long runs")


def test_shared_and_weighted_in_one_graph_on_a_side_stream():
    """Both passes behind one another in one captured graph on a stream of its own, replayed with other lengths that share
    nothing any more."""
    seq = [900 + 40 * i for i in range(5)]
    prob = make_problem(61, 2, 5, 8, 2, 128, seq)
    share_prefixes(prob, [0, 5], [899])
    ctx = gh.make_ctx(prob, [64] * 2, [4] * 2, [1] * 2)
    dev = gh.upload(prob)
    i32 = dict(dtype=torch.int32, device="cuda")
    gs, gp, f = torch.tensor([0, 5], **i32), torch.tensor([899], **i32), torch.ones(5, **ONES)
    out, lse = gh.new_out(prob, fill=-3.0)
    out2, lse2 = gh.new_out(prob, fill=-3.0)
    w = torch.zeros((2, 5, 2, prob["table"].shape[1] * 16), device="cuda")
    side = torch.cuda.Stream()
    s1, s2 = ctx.full_decode_shared_scratch(), ctx.full_decode_weighted_scratch()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        ctx.full_decode_shared(0, 2, 5, dev["q"], dev["k"], dev["v"], dev["table"], dev["seq_lens"], f, gs, gp, out, lse, scratch=s1)
        ctx.full_decode_weighted(0, 2, 5, dev["q"], dev["k"], dev["v"], dev["table"], dev["seq_lens"], f, w, out2, lse2, scratch=s2)
    with torch.cuda.stream(side):
        g.replay()
    side.synchronize()
    ref, rlse, _ = full_reference(prob)
    rows_close(out, lse, ref, rlse, [0, 1], range(5), "shared")
    rows_close(out2, lse2, ref, rlse, [0, 1], range(5), "weighted")
    dev["seq_lens"].copy_(torch.tensor([1, 17, 900, 64, 1060]))
    gp.copy_(torch.tensor([0]))
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        g.replay()
    side.synchronize()
    ref, rlse, _ = full_reference(dict(prob, seq_lens=np.array([1, 17, 900, 64, 1060], np.int32)))
    rows_close(out, lse, ref, rlse, [0, 1], range(5), "shared, replayed")
    rows_close(out2, lse2, ref, rlse, [0, 1], range(5), "weighted, replayed")
    assert ctx.read_device_status() == 0


def test_shared_one_tile_of_two_blocks_of_rows_many_times():
    """Prefixes of one tile whose rows are a block for both row tiles and a rest for one: a CTA changes between the two kinds
    of item at every tile, and no stream may be ahead of the other across the change.  Against the plain gated pass, and
    the same bits every time."""
    L, B, Hq, Hkv, D = 96, 99, 64, 8, 64
    seq = [64 + 1 + i % 9 for i in range(B)]
    prob = make_problem(62, 1, B, Hq, Hkv, D, seq)
    share_prefixes(prob, [0, 33, 66, 99], [64] * 3)
    prob = dict(prob, L=L, q=synth.gauss_bf16_tensor(63, synth.STREAM_Q, (L, B, Hq, D)))
    ctx = gh.make_ctx(prob, [16] * L, [0] * L, [1] * L, kv_index=[0] * L)
    dev = gh.upload(prob)
    f = torch.ones(B, **ONES)
    want, wlse = gh.new_out(prob)
    ctx.full_decode_gated(0, L, B, dev["q"], dev["k"], dev["v"], dev["table"], dev["seq_lens"], f, want, wlse)
    first = None
    for _ in range(40):
        _, out, lse = run_shared(prob, [0, 33, 66, 99], [64] * 3, [1] * B, ctx=ctx, dev=dev)
        if first is None:
            first = (out, lse)
            assert (out - want).abs().max() <= gh.ATOL_OUT and (lse - wlse).abs().max() <= gh.ATOL_LSE
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    assert ctx.read_device_status() == 0
