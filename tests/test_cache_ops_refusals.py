"""What the shared-prefix pass, the weighted pass and the eviction refuse, checked on the host without a device."""
import pytest
import torch

from paper_2609_20734_b200 import binding
from tests.test_abi import base_cfg

LIB = binding.load_library()


def ctx_of(**kw):
    return binding.OdaContext(base_cfg(**kw), allocate_workspace=False)


def refused(status, call, *args, **kw):
    with pytest.raises(binding.OdaError) as e:
        call(*args, **kw)
    assert e.value.status == status, str(e.value)


def test_null_context():
    assert LIB.oda_full_decode_shared(None, 0, 1, 1, *[None] * 6, 0, *[None] * 5, 0, None) == 1
    assert LIB.oda_full_decode_weighted(None, 0, 1, 1, *[None] * 10, 0, None) == 1
    assert LIB.oda_evict(None, 1, *[None] * 6, 1, 0, 0, None, None, 0, None) == 1
    assert LIB.oda_full_decode_shared_scratch_bytes(None) == 0
    assert LIB.oda_full_decode_weighted_scratch_bytes(None, 1, 1) == 0
    assert LIB.oda_evict_scratch_bytes(None) == 0


def test_scratch_sizes():
    ctx = ctx_of()
    one = LIB.oda_full_decode_weighted_scratch_bytes(ctx._h, 1, 4)
    assert one >= 4 * 8 * 64 * 16 * 4 and one % 256 == 0
    assert LIB.oda_full_decode_weighted_scratch_bytes(ctx._h, 2, 4) == 2 * one
    assert LIB.oda_full_decode_weighted_scratch_bytes(ctx._h, 3, 4) == 0      # more layers than the context has
    assert LIB.oda_full_decode_weighted_scratch_bytes(ctx._h, 1, 5) == 0      # more requests
    assert LIB.oda_evict_scratch_bytes(ctx._h) == 2 * 4 * 2 * 64 * 16 * 4
    assert LIB.oda_full_decode_shared_scratch_bytes(ctx._h) > 0
    aliased = ctx_of(layer_kv_index=[0, 0])
    assert aliased.kv_slices == 1 and LIB.oda_evict_scratch_bytes(aliased._h) == 4 * 2 * 64 * 16 * 4


def fake(n, dtype=torch.float32):
    return torch.empty(n, dtype=dtype)


def evict(ctx, batch=4, budget=64, sinks=4, recent=16, kept=None, **kw):
    w = fake(2 * 4 * 2 * 64 * 16)
    return ctx.evict(batch, w, 256, 256, 256, 256, budget, sinks, recent, kept=kept, scratch=fake(4, torch.uint8), stream=0, **kw)


@pytest.mark.parametrize("kw", [dict(budget=0), dict(budget=64 * 16 + 1), dict(budget=-1), dict(sinks=-1), dict(recent=-1),
                                dict(sinks=40, recent=25), dict(sinks=2**31 - 1, recent=2**31 - 1), dict(batch=5), dict(batch=-1)])
def test_evict_refuses_bad_arguments(kw):
    refused(1, evict, ctx_of(), **kw)


def test_evict_needs_a_workspace_and_tensors_of_the_right_size():
    ctx = ctx_of()
    refused(3, evict, ctx)
    with pytest.raises(ValueError):
        ctx.evict(4, fake(10), 256, 256, 256, 256, 64, 0, 0, stream=0)
    with pytest.raises(ValueError):
        evict(ctx, kept=fake(7, torch.int32))
    with pytest.raises(ValueError):
        evict(ctx, kept=fake(2 * 4 * 2 * 64, torch.int64))


def test_passes_need_a_workspace_and_matching_groups():
    ctx = ctx_of()
    w = fake(2 * 4 * 2 * 64 * 16)
    s = fake(256, torch.uint8)
    refused(3, ctx.full_decode_weighted, 0, 2, 1, 256, 256, 256, 256, 256, 256, w, 256, None, scratch=s, stream=0)
    refused(3, ctx.full_decode_shared, 0, 2, 1, 256, 256, 256, 256, 256, 256, None, None, 256, None, scratch=s, stream=0)
    with pytest.raises(ValueError):
        ctx.full_decode_weighted(0, 2, 1, 256, 256, 256, 256, 256, 256, fake(5), 256, None, scratch=s, stream=0)
    with pytest.raises(ValueError):
        ctx.full_decode_shared(0, 2, 2, 256, 256, 256, 256, 256, 256, fake(2, torch.int32), fake(2, torch.int32), 256, None,
                               scratch=s, stream=0)
    with pytest.raises(ValueError):
        ctx.full_decode_shared(0, 2, 2, 256, 256, 256, 256, 256, 256, fake(2, torch.int64), fake(1, torch.int64), 256, None,
                               scratch=s, stream=0)


@pytest.mark.gpu
def test_refusals_behind_the_workspace():
    """Null and misaligned pointers, missing scratch, the variant without these passes: nothing is launched."""
    ctx = binding.OdaContext(base_cfg())
    n = ctx.launch_count
    w = torch.zeros(2 * 4 * 2 * 64 * 16, device="cuda")
    big = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    i32 = torch.zeros(16, dtype=torch.int32, device="cuda")
    p = big.data_ptr()
    weighted = lambda **k: ctx.full_decode_weighted(*[{**dict(lb=0, le=2, b=4, q=p, k=p, v=p, t=p, s=p, f=p, w=w, o=p, l=None), **k}[x]  # noqa: E731
                                                      for x in ("lb", "le", "b", "q", "k", "v", "t", "s", "f", "w", "o", "l")],
                                                    scratch=k.get("scratch", big))
    shared = lambda **k: ctx.full_decode_shared(*[{**dict(lb=0, le=2, b=4, q=p, k=p, v=p, t=p, s=p, f=p, gs=i32[:2], gp=i32[:1], o=p, l=None), **k}[x]  # noqa: E731
                                                  for x in ("lb", "le", "b", "q", "k", "v", "t", "s", "f", "gs", "gp", "o", "l")],
                                                scratch=k.get("scratch", big))
    for call in (weighted, shared):
        for bad in (dict(q=None), dict(k=None), dict(t=None), dict(s=None), dict(f=None), dict(o=None), dict(q=p + 8), dict(v=p + 2),
                    dict(lb=-1), dict(le=3), dict(lb=2, le=1), dict(b=5), dict(b=-1)):
            refused(1, call, **bad)
        for bad in (dict(scratch=big[:16]), dict(scratch=big[1:])):
            refused(3, call, **bad)
    refused(1, shared, gs=torch.zeros(130, dtype=torch.int32, device="cuda"), gp=torch.zeros(129, dtype=torch.int32, device="cuda"))
    for bad in (dict(k_cache=None), dict(v_cache=p + 8), dict(block_table=None), dict(seq_lens=None)):
        a = dict(k_cache=p, v_cache=p, block_table=p, seq_lens=p, **{})
        a.update(bad)
        refused(1, ctx.evict, 4, w, a["k_cache"], a["v_cache"], a["block_table"], a["seq_lens"], 64, 0, 0, scratch=big)
    refused(3, ctx.evict, 4, w, p, p, p, p, 64, 0, 0, scratch=big[:64])
    simt = binding.OdaContext(base_cfg(variant=binding.VARIANT_SIMT))
    refused(2, simt.full_decode_weighted, 0, 2, 4, p, p, p, p, p, p, w, p, None, scratch=big)
    refused(2, simt.full_decode_shared, 0, 2, 4, p, p, p, p, p, p, i32[:2], i32[:1], p, None, scratch=big)
    assert ctx.launch_count == n and simt.launch_count == 0
    # nothing to do: no launch, no error
    ctx.full_decode_shared(0, 2, 0, None, None, None, None, None, None, None, None, None, None, scratch=big)
    ctx.full_decode_weighted(1, 1, 4, None, None, None, None, None, None, w, None, None, scratch=big)
    ctx.evict(0, w, None, None, None, None, 64, scratch=big)
    assert ctx.launch_count == n
