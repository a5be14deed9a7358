"""Cases of three operators over the paged decode cache, with their plain forms.

  shared    the gated Full pass for requests that begin with the same prefix (`full_decode_shared`)
  weighted  the gated Full pass that also adds up the attention weight of every position (`full_decode_weighted`)
  evict     dropping the lightest positions of a cache down to a budget (`evict`)

Caches are bf16 pages of 16 positions behind a block table, [slices, blocks, kv heads, 16, D] ("hnd") or
[slices, blocks, 16, kv heads, D] ("nhd").  `own` says whose work `run` does: the plain forms below, or the calls of
this repository's binding.
"""
import math

import numpy as np
import torch

own = False

P = 16  # positions of a page


# ---------------------------------------------------------------------------------------------- the cases
def listed():
    return [
        # one layer of a model with 4 requests behind a 2K system prompt: a call in which latency counts
        dict(name="shared_layer_b4", op="shared", L=1, B=4, Hq=32, Hkv=8, D=128, layout="hnd", out="bf16",
             groups=1, prefix=2048, tail_lo=17, tail_hi=200, flagged=100),
        # the 32-layer configuration, 16 requests about one document of odd length, tails of a dialogue
        dict(name="shared_32l_b16", op="shared", L=32, B=16, Hq=32, Hkv=8, D=128, layout="hnd", out="bf16",
             groups=1, prefix=8197, tail_lo=1, tail_hi=1000, flagged=100),
        # heads of the 64/8 configuration, 64 samples drawn from one long prompt: 512 query rows a kv head
        dict(name="shared_g8_b64", op="shared", L=8, B=64, Hq=64, Hkv=8, D=128, layout="hnd", out="bf16",
             groups=1, prefix=32768, tail_lo=30, tail_hi=333, flagged=100),
        # three prompts in one batch, some requests not recalled, small heads, fp32 results, the other layout
        dict(name="shared_groups_d64", op="shared", L=6, B=24, Hq=16, Hkv=8, D=64, layout="nhd", out="fp32",
             groups=3, prefix=5003, tail_lo=1, tail_hi=700, flagged=75),
        # one layer of a short history: a call in which latency counts
        dict(name="weighted_layer_2k", op="weighted", L=1, B=1, Hq=32, Hkv=8, D=128, layout="hnd", out="bf16",
             len_lo=2049, len_hi=2049, flagged=100),
        # a recalled step of the 32-layer configuration at 32,768 tokens
        dict(name="weighted_32l_32k", op="weighted", L=32, B=1, Hq=32, Hkv=8, D=128, layout="hnd", out="bf16",
             len_lo=32768, len_hi=32768, flagged=100),
        # a ragged batch with heads of the 64/8 configuration, half of it recalled, fp32 results
        dict(name="weighted_ragged_g8", op="weighted", L=8, B=16, Hq=64, Hkv=8, D=128, layout="nhd", out="fp32",
             len_lo=1, len_hi=16384, flagged=50),
        # one position too many after a step: the running form of a fixed budget, one layer
        dict(name="evict_step_layer", op="evict", L=1, B=2, Hkv=8, D=128, layout="hnd",
             len_lo=2053, len_hi=2053, budget=2052, sinks=4, recent=1024),
        # the 32-layer configuration from 32,768 tokens down to a quarter
        dict(name="evict_32l_32k", op="evict", L=32, B=1, Hkv=8, D=128, layout="hnd",
             len_lo=32768, len_hi=32768, budget=8192, sinks=4, recent=1024),
        # a ragged batch, some requests within the budget, small heads, the other layout
        dict(name="evict_ragged_d64", op="evict", L=8, B=16, Hkv=8, D=64, layout="nhd",
             len_lo=700, len_hi=9000, budget=4001, sinks=4, recent=512),
        # few heads over a very long history (a card of a head-parallel group)
        dict(name="evict_long_1l", op="evict", L=1, B=1, Hkv=8, D=128, layout="hnd",
             len_lo=262144, len_hi=262144, budget=65536, sinks=4, recent=2048),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(("shared", "weighted", "evict"))
    D = rng.choice((64, 128, 128))
    Hkv = rng.choice((1, 2, 4, 8))
    layout = rng.choice(("hnd", "nhd"))
    if op == "evict":
        t = _log_int(rng, 200, 40000)
        B = _log_int(rng, 1, 16)
        L = _log_int(rng, 1, max(1, min(32, 8_000_000 // (t * B * Hkv))))
        sinks = rng.choice((0, 1, 4, 17))
        recent = _log_int(rng, 1, max(1, t // 4))
        budget = min(t, max(sinks + recent, _log_int(rng, max(1, t // 16), t)))
        return dict(op=op, L=L, B=B, Hkv=Hkv, D=D, layout=layout, len_lo=max(1, t // rng.choice((1, 1, 2, 5))), len_hi=t,
                    budget=budget, sinks=sinks, recent=recent)
    G = rng.choice((1, 2, 4, 8))
    out = rng.choice(("bf16", "fp32"))
    flagged = rng.choice((100, 100, 60))
    if op == "weighted":
        t = _log_int(rng, 16, 40000)
        B = _log_int(rng, 1, 24)
        L = _log_int(rng, 1, max(1, min(32, 4_000_000 // (t * B * Hkv))))
        return dict(op=op, L=L, B=B, Hq=Hkv * G, Hkv=Hkv, D=D, layout=layout, out=out, len_lo=max(1, t // rng.choice((1, 3, 50))),
                    len_hi=t, flagged=flagged)
    groups = rng.choice((1, 1, 2, 4))
    B = groups * _log_int(rng, 2, 96 // groups)
    prefix = _log_int(rng, 40, 30000)
    tail = _log_int(rng, 2, 1500)
    L = _log_int(rng, 1, max(1, min(32, 3_000_000 // ((prefix * groups + tail * B) * Hkv))))
    return dict(op=op, L=L, B=B, Hq=Hkv * G, Hkv=Hkv, D=D, layout=layout, out=out, groups=groups, prefix=prefix,
                tail_lo=rng.choice((1, max(1, tail // 4))), tail_hi=tail, flagged=flagged)


# ---------------------------------------------------------------------------------------------- inputs
def _lengths(case, rs):
    lo, hi = case["len_lo"], case["len_hi"]
    t = rs.randint(lo, hi + 1, case["B"])
    t[rs.randint(case["B"])] = hi  # the longest is there
    return t.astype(np.int32)


def _flags(case, rs):
    f = (rs.rand(case["B"]) * 100 < case["flagged"]).astype(np.uint8)
    f[0] = 1
    return f


def _cache(case, blocks, gen, heavy):
    """Random keys or values; `heavy`: one key in 96 is longer, as those of sinks and names are."""
    L, H, D = case["L"], case["Hkv"], case["D"]
    shape = (L, blocks, H, P, D) if case["layout"] == "hnd" else (L, blocks, P, H, D)
    c = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    if heavy:
        if case["layout"] == "hnd":
            c[:, ::6, :, 5] *= 2.5
        else:
            c[:, ::6, 5] *= 2.5
    return c


def _context(case, state, window=1024, sinks=4):
    """The handle that a user's program keeps for its model."""
    from paper_2609_20734_b200.binding import OdaConfig, OdaContext

    L, H, D, blocks = case["L"], case["Hkv"], case["D"], state["k"].shape[1]
    hnd = case["layout"] == "hnd"
    return OdaContext(OdaConfig(
        num_layers=L, num_q_heads=case.get("Hq", H), num_kv_heads=H, head_dim=D, max_batch=case["B"],
        max_blocks_per_seq=state["table"].shape[1], layer_window=[window] * L, layer_sinks=[sinks] * L,
        layer_gated=[1] * L, kv_layer_stride=blocks * H * P * D, kv_block_stride=H * P * D,
        kv_token_stride=D if hnd else H * D, kv_head_stride=P * D if hnd else D,
        out_dtype=1 if case.get("out") == "bf16" else 0))


def _attention_state(case, lens, table, blocks, rs, gen):
    L, B, Hq, D = case["L"], case["B"], case["Hq"], case["D"]
    dt = torch.bfloat16 if case["out"] == "bf16" else torch.float32
    s = dict(case=case, table=torch.from_numpy(table).cuda(), seq_lens=torch.from_numpy(lens).cuda(),
             flags=torch.from_numpy(_flags(case, rs)).cuda())
    s["k"] = _cache(case, blocks, gen, True)
    s["v"] = _cache(case, blocks, gen, False)
    s["q"] = torch.empty((L, B, Hq, D), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    # what the Local pass left there: rows of requests that are not flagged keep it
    s["out"] = torch.empty((L, B, Hq, D), dtype=dt, device="cuda").normal_(generator=gen)
    s["lse"] = torch.empty((L, B, Hq), dtype=torch.float32, device="cuda").normal_(generator=gen)
    return s


def prepare(case, seed):
    rs = np.random.RandomState(seed % (1 << 31))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    B = case["B"]
    if case["op"] == "shared":
        # requests in order of their groups; pages before the prefix's last whole page are one and the same
        cut = [B * g // case["groups"] for g in range(case["groups"] + 1)]
        prefix = [max(1, case["prefix"] - 37 * g) for g in range(case["groups"])]
        of = np.repeat(np.arange(case["groups"]), np.diff(cut))
        tail = rs.randint(case["tail_lo"], case["tail_hi"] + 1, B)
        lens = np.array([prefix[g] for g in of], np.int32) + tail.astype(np.int32)
        whole = [p // P for p in prefix]
        pages = [(int(t) + P - 1) // P for t in lens]
        blocks = sum(whole) + sum(n - whole[g] for n, g in zip(pages, of))
        ids = rs.permutation(blocks).astype(np.int32)
        table = np.zeros((B, max(pages)), np.int32)
        at, first = 0, {}
        for b in range(B):
            g = int(of[b])
            if g not in first:
                first[g] = ids[at:at + whole[g]]
                at += whole[g]
            n = pages[b] - whole[g]
            table[b, :whole[g]] = first[g]
            table[b, whole[g]:pages[b]] = ids[at:at + n]
            at += n
        s = _attention_state(case, lens, table, blocks, rs, gen)
        for b in range(B):  # a prefix that ends inside a page: every request has its own copy of that page's beginning
            g = int(of[b])
            r, lead = prefix[g] % P, cut[g]
            if r and b != lead:
                src, dst = int(table[lead, whole[g]]), int(table[b, whole[g]])
                for c in (s["k"], s["v"]):
                    if case["layout"] == "hnd":
                        c[:, dst, :, :r] = c[:, src, :, :r]
                    else:
                        c[:, dst, :r] = c[:, src, :r]
        s["cut"], s["prefix"] = cut, prefix
        s["group_start"] = torch.tensor(cut, dtype=torch.int32, device="cuda")
        s["group_prefix"] = torch.tensor(prefix, dtype=torch.int32, device="cuda")
    else:
        lens = _lengths(case, rs)
        pages = [(int(t) + P - 1) // P for t in lens]
        width = max(pages)
        blocks = B * width  # what the pool has room for, whatever the lengths are
        ids = rs.permutation(blocks).astype(np.int32)
        table, at = np.zeros((B, width), np.int32), 0
        for b in range(B):
            table[b, :pages[b]] = ids[at:at + pages[b]]
            at += pages[b]
        shape = (case["L"], B, case["Hkv"], width * P)
        if case["op"] == "weighted":
            s = _attention_state(case, lens, table, blocks, rs, gen)
            s["weights"] = torch.empty(shape, dtype=torch.float32, device="cuda").exponential_(generator=gen) * 1e-3
        else:
            s = dict(case=case, table=torch.from_numpy(table).cuda(), lens0=torch.from_numpy(lens).cuda())
            s["k"] = _cache(case, blocks, gen, True)
            s["v"] = _cache(case, blocks, gen, False)
            # few heavy positions, many light ones, some of equal weight and some that were never looked at
            w = torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=gen).mul_(2).exp_()
            w = torch.where(w < 0.2, torch.zeros_like(w), torch.where(w < 1, (w * 64).floor() / 64, w))
            s["weights0"], s["weights"] = w, torch.empty_like(w)
            s["seq_lens"] = torch.empty_like(s["lens0"])
            s["kept"] = torch.empty((case["L"], B, case["Hkv"], case["budget"]), dtype=torch.int32, device="cuda")
    s["ctx"] = _context(case, s) if own else None
    if own:
        make = dict(shared="full_decode_shared_scratch", weighted="full_decode_weighted_scratch", evict="evict_scratch")
        s["scratch"] = getattr(s["ctx"], make[case["op"]])()
    return s


# ---------------------------------------------------------------------------------------------- plain forms
def _pages(cache, layout, layer, blocks):
    """Rows of the pages `blocks` [..., n] of one layer: fp32 [..., kv heads, n * 16, D]."""
    x = cache[layer][blocks.long()].float()
    x = x.movedim(-3, -4) if layout == "hnd" else x.movedim(-2, -4)  # [..., H, n, 16, D]
    return x.flatten(-3, -2)


def _plain_shared(s):
    case = s["case"]
    G, H, D, lay = case["Hq"] // case["Hkv"], case["Hkv"], case["D"], case["layout"]
    scale = 1.0 / math.sqrt(D)
    take = s["flags"].bool()
    for layer in range(case["L"]):
        for g, n0 in enumerate(s["prefix"]):
            b0, b1 = s["cut"][g], s["cut"][g + 1]
            n, full = b1 - b0, (n0 + P - 1) // P
            q = s["q"][layer, b0:b1].float().view(n, H, G, D) * scale
            # the prefix, once for all requests of the group
            kp = _pages(s["k"], lay, layer, s["table"][b0, :full])[:, :n0]
            vp = _pages(s["v"], lay, layer, s["table"][b0, :full])[:, :n0]
            zp = (q.transpose(0, 1).reshape(H, n * G, D) @ kp.transpose(1, 2)).view(H, n, G, n0).transpose(0, 1)
            # each request's tail
            first = n0 // P
            ks = _pages(s["k"], lay, layer, s["table"][b0:b1, first:])
            vs = _pages(s["v"], lay, layer, s["table"][b0:b1, first:])
            zs = q @ ks.transpose(2, 3)
            pos = first * P + torch.arange(zs.shape[-1], device=q.device)
            here = (pos >= n0) & (pos < s["seq_lens"][b0:b1, None])
            zs = torch.where(here[:, None, None], zs, float("-inf"))
            m = torch.maximum(zp.amax(-1, keepdim=True), zs.amax(-1, keepdim=True))
            wp, ws = (zp - m).exp(), (zs - m).exp()
            den = wp.sum(-1, keepdim=True) + ws.sum(-1, keepdim=True)
            top = (wp.transpose(0, 1).reshape(H, n * G, n0) @ vp).view(H, n, G, D).transpose(0, 1) + ws @ vs
            o = (top / den).reshape(n, H * G, D).to(s["out"].dtype)
            e = (m + den.log()).reshape(n, H * G)
            f = take[b0:b1, None]
            s["out"][layer, b0:b1] = torch.where(f[..., None], o, s["out"][layer, b0:b1])
            s["lse"][layer, b0:b1] = torch.where(f, e, s["lse"][layer, b0:b1])
    return s["out"], s["lse"]


def _plain_weighted(s):
    case = s["case"]
    B, G, H, D, lay = case["B"], case["Hq"] // case["Hkv"], case["Hkv"], case["D"], case["layout"]
    scale = 1.0 / math.sqrt(D)
    take = s["flags"].bool()
    for layer in range(case["L"]):
        q = s["q"][layer].float().view(B, H, G, D) * scale
        k = _pages(s["k"], lay, layer, s["table"])
        v = _pages(s["v"], lay, layer, s["table"])
        z = q @ k.transpose(2, 3)
        here = torch.arange(z.shape[-1], device=q.device) < s["seq_lens"][:, None]
        z = torch.where(here[:, None, None], z, float("-inf"))
        m = z.amax(-1, keepdim=True)
        w = (z - m).exp()
        den = w.sum(-1, keepdim=True)
        w = w / den
        o = (w @ v).reshape(B, H * G, D).to(s["out"].dtype)
        e = (m + den.log()).reshape(B, H * G)
        s["out"][layer] = torch.where(take[:, None, None], o, s["out"][layer])
        s["lse"][layer] = torch.where(take[:, None], e, s["lse"][layer])
        s["weights"][layer] += torch.where(take[:, None, None], w.sum(2), torch.zeros((), device=q.device))
    return s["out"], s["lse"], s["weights"]


def _plain_evict(s):
    case = s["case"]
    L, B, H, n, most = case["L"], case["B"], case["Hkv"], case["budget"], s["weights"].shape[-1]
    t = s["seq_lens"].view(B, 1, 1).long()
    pos = torch.arange(most, device=t.device)
    w = s["weights"]
    key = torch.where((pos < case["sinks"]) | (pos >= t - case["recent"]), float("inf"), w)
    key = torch.where(pos < t, key, float("-inf"))
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :n].sort(-1).values
    i = torch.arange(n, device=t.device)
    order = torch.where(t > n, order, i)                        # within the budget: nothing moves
    there = i < t
    # rows behind a short request's end: its row 0 once more, onto itself
    src = torch.where(there, order, 0)
    dst = torch.where(there, i, 0).expand(L, B, H, n)
    table = s["table"].long()
    a = (torch.arange(L, device=t.device).view(L, 1, 1, 1), torch.arange(B, device=t.device).view(1, B, 1, 1),
         torch.arange(H, device=t.device).view(1, 1, H, 1))
    for c in (s["k"], s["v"]):
        x = c if case["layout"] == "hnd" else c.transpose(2, 3)
        x[a[0], table[a[1], dst // P], a[2], dst % P] = x[a[0], table[a[1], src // P], a[2], src % P]
    moved = torch.where(there, w.gather(-1, src), torch.zeros((), device=t.device))
    new = torch.where(pos < n, 0, torch.where(pos < t, torch.zeros((), device=t.device), w))
    new[..., :n] = torch.where(there, moved, w[..., :n])
    w.copy_(new)
    s["kept"].copy_(torch.where(there, order, -1))
    s["seq_lens"].copy_(torch.minimum(s["seq_lens"], torch.full_like(s["seq_lens"], n)))
    return s["k"], s["v"], s["weights"], s["seq_lens"], s["kept"]


def run(s):
    case = s["case"]
    if case["op"] == "evict":  # the state before the eviction: a pass can be repeated on rows that it has moved
        s["weights"].copy_(s["weights0"])
        s["seq_lens"].copy_(s["lens0"])
    if not own:
        return dict(shared=_plain_shared, weighted=_plain_weighted, evict=_plain_evict)[case["op"]](s)
    ctx = s["ctx"]
    if case["op"] == "shared":
        ctx.full_decode_shared(0, case["L"], case["B"], s["q"], s["k"], s["v"], s["table"], s["seq_lens"], s["flags"],
                               s["group_start"], s["group_prefix"], s["out"], s["lse"], scratch=s["scratch"])
        return s["out"], s["lse"]
    if case["op"] == "weighted":
        ctx.full_decode_weighted(0, case["L"], case["B"], s["q"], s["k"], s["v"], s["table"], s["seq_lens"], s["flags"],
                                 s["weights"], s["out"], s["lse"], scratch=s["scratch"])
        return s["out"], s["lse"], s["weights"]
    ctx.evict(case["B"], s["weights"], s["k"], s["v"], s["table"], s["seq_lens"], case["budget"], case["sinks"],
              case["recent"], kept=s["kept"], scratch=s["scratch"])
    return s["k"], s["v"], s["weights"], s["seq_lens"], s["kept"]


# ---------------------------------------------------------------------------------------------- work and exact values
def _mean_len(case):
    """Expected sum of a batch's lengths (one of them is the longest)."""
    return case["len_hi"] + (case["B"] - 1) * (case["len_lo"] + case["len_hi"]) / 2


def work(case):
    L, B, H, D = case["L"], case["B"], case["Hkv"], case["D"]
    row = 2 * D * 2  # K and V of one position and kv head
    if case["op"] == "evict":
        n = case["budget"]
        # requests over the budget; of their kept rows, those behind the first dropped one move
        span = max(1, case["len_hi"] - case["len_lo"] + 1)
        over = 1 + (B - 1) * max(0, case["len_hi"] - max(n, case["len_lo"] - 1)) / span if case["len_hi"] > n else 0
        long = (max(n, case["len_lo"]) + case["len_hi"]) / 2
        dropped = max(1, long - n)
        still = case["sinks"] + max(0, n - case["sinks"] - case["recent"]) / (dropped + 1)
        units = L * H
        return dict(bytes=units * (over * (max(0, n - still) * row * 2 + long * 4 + n * 8) + (B - over) * n * 4), flops=units * over * long)
    Hq, ob = case["Hq"], 2 if case["out"] == "bf16" else 4
    share = case["flagged"] / 100
    io = L * B * share * Hq * (D * 2 + D * ob + 4)
    if case["op"] == "shared":
        prefix = sum(max(1, case["prefix"] - 37 * g) for g in range(case["groups"]))
        tail = (case["tail_lo"] + case["tail_hi"]) / 2 * B * share
        seen = tail + prefix / case["groups"] * B * share
        return dict(bytes=L * H * row * (prefix + tail) + io, flops=4 * D * L * Hq * seen)
    seen = _mean_len(case) * share
    return dict(bytes=L * H * seen * (row + 8) + io, flops=4 * D * L * Hq * seen)


def _dense(cache, layout, layer, blocks, t):
    """fp64 [kv heads, t, D] of one request's layer."""
    x = cache[layer][blocks[: (t + P - 1) // P].long()].double()
    x = x.permute(1, 0, 2, 3) if layout == "hnd" else x.permute(2, 0, 1, 3)
    return x.reshape(x.shape[0], -1, x.shape[-1])[:, :t]


def exact(case, seed):
    s = prepare(case, seed)
    H, D, lay = case["Hkv"], case["D"], case["layout"]
    if case["op"] != "evict":
        G = case["Hq"] // H
        out, lse = s["out"].double(), s["lse"].double()
        acc = s["weights"].double() if case["op"] == "weighted" else None
        lens, flags = s["seq_lens"].tolist(), s["flags"].tolist()
        for b in range(case["B"]):
            if not flags[b]:
                continue
            t = lens[b]
            for layer in range(case["L"]):
                k, v = _dense(s["k"], lay, layer, s["table"][b], t), _dense(s["v"], lay, layer, s["table"][b], t)
                q = s["q"][layer, b].double().view(H, G, D)
                z = torch.bmm(q, k.transpose(1, 2)) / math.sqrt(D)
                e = torch.logsumexp(z, -1)
                w = torch.exp(z - e[..., None])
                out[layer, b] = torch.bmm(w, v).reshape(H * G, D)
                lse[layer, b] = e.reshape(H * G)
                if acc is not None:
                    acc[layer, b, :, :t] += w.sum(1)
        return (out, lse) if acc is None else (out, lse, acc)
    # eviction: every (slice, request, head) by itself, on the host
    n, w0 = case["budget"], s["weights0"].double().cpu().numpy()
    lens, table = s["lens0"].tolist(), s["table"].cpu().numpy()
    new, kept = w0.copy(), np.full(s["kept"].shape, -1, np.int64)
    for b, t in enumerate(lens):
        for layer in range(case["L"]):
            for h in range(H):
                if t <= n:
                    kept[layer, b, h, :t] = np.arange(t)
                    continue
                lo, hi = case["sinks"], t - case["recent"]
                mid = w0[layer, b, h, lo:hi]
                best = lo + np.lexsort((np.arange(hi - lo), -mid))[: n - case["sinks"] - case["recent"]]
                keep = np.concatenate([np.arange(lo), np.sort(best), np.arange(hi, t)])
                kept[layer, b, h] = keep
                new[layer, b, h, :n] = w0[layer, b, h, keep]
                new[layer, b, h, n:t] = 0
                old = torch.from_numpy(keep).cuda()
                to = torch.from_numpy(table[b]).cuda().long()
                i = torch.arange(n, device="cuda")
                for c in (s["k"], s["v"]):
                    x = c[layer, :, h] if lay == "hnd" else c[layer, :, :, h]
                    x[to[i // P], i % P] = x[to[old // P], old % P].clone()
    lens = torch.tensor([min(t, n) for t in lens], dtype=torch.int32, device="cuda")
    return s["k"], s["v"], torch.from_numpy(new).cuda(), lens, torch.from_numpy(kept).cuda()
