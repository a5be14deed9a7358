// Attention of many requests over a prefix that they share, on the 5th-generation tensor cores.
//
// The gated Full pass over shared prefixes is two launches.  This kernel does the shared part: for every (gated
// layer, kv head, group of requests) the query heads of all flagged requests of the group are the rows of one
// matrix Q, and
//     S = Q K^T,  P = 2^(scale S - m),  O = P V,  l = P 1
// runs over the prefix once.  What is left of each request -- its own tail of positions -- goes to the split-KV
// kernel, whose epilogue folds the partial results of this kernel in (SharedDesc says where they are).
//
// Only whole pages are shared (a page that the prefix ends in is read through each request's own table row), and
// every request keeps at least one position of its own, so the second kernel visits every flagged request.
//
// Work: rows are cut into blocks of 256 (two 128-row MMA tiles), prefixes into tiles of kTokens positions; all
// (layer, kv head, group, row block, tile) lie on one axis that is cut into equal spans, one per CTA (one CTA per SM).
// A unit that a span boundary cuts leaves several partials; nobody waits for another CTA.
//
// A CTA: two softmax warpgroups ("streams"), one producer warp (TMA), one MMA warp (one thread issues).  With more than
// 128 rows the streams are the two row tiles and both use every K/V tile; with fewer, both have the same rows and take
// the tiles in turn (stream 0 the even ones), and their results are joined through TMEM at the end.  Either way one
// stream's softmax runs while the tensor core works for the other.  TMEM: S of both streams (kTokens columns each; P
// replaces S in place as bf16) and O of both streams (D columns each).
//
// P in bf16: kTerms parts of 8 bits each.  Three for fp32 results (24 bits: nothing is lost against fp32 arithmetic);
// for bf16 results see launch_shared_prefix.
#include <cuda.h>

#include "launch_ex.cuh"
#include "mbar.cuh"
#include "oda_device.cuh"
#include "oda_launch.h"
#include "shared_prefix.cuh"

namespace oda {

constexpr int kShThreads = 320;
constexpr int kShRows = 128;       // rows of one MMA tile
constexpr int kShMinTiles = 2;     // a CTA is not given fewer tiles than this (unless there are fewer)

template <int D, int kTerms>
struct ShCfg {
    static constexpr int kTokens = kTerms == 3 ? 64 : 128;  // S (and three parts of P) of two streams beside O in 512 columns
    static constexpr int kTilePages = kTokens / kPage;
    static constexpr int kSlotBytes = kTokens * D * 2;      // K or V of one tile
    static constexpr int kSlots = 131072 / kSlotBytes > 16 ? 16 : 131072 / kSlotBytes;
    static constexpr int kQBytes = kShRows * D * 2;
    static constexpr int kSpCols = kTerms == 3 ? 96 : kTokens;  // columns of one stream's S and P
    static constexpr int kO0 = 2 * kSpCols;                 // first column of stream 0's O
    static_assert(2 * kSpCols + 2 * D <= 512, "TMEM");
};

struct ShPlan {
    int32_t t[kMaxBatch];            // lengths, clamped to the table
    int32_t gs[kMaxBatch + 1];
    int32_t off[kMaxBatch + 1];      // first tile of each group within one (layer, kv head)
    int32_t pages[kMaxBatch];        // shared pages of the group (0: shares nothing)
    uint8_t members[kMaxBatch];      // flagged ones of each group
    uint8_t act[kMaxBatch];
    uint8_t list[kMaxBatch];         // flagged requests, those of group i from gs[i] on
    int32_t t1, total, nseg;
};

struct ShCtl {
    uint64_t full[16], empty[16];
    uint64_t s_full[2], p_full[2], o_full[2], q_full[2];
    uint64_t ml_full, o1_read;       // joining the streams: stream 1's (m, l) are there, its O has been read
    uint32_t tmem;
    int32_t abort;
    float2 ml1[kShRows];             // stream 1's (m, l) when the streams are joined
};

struct ShItem {
    int32_t gl, kvh, group, row0, nrows, tile0, n, pages;  // gated layer index, ..., first row, rows, first tile, tiles, pages of the prefix
};

// ------------------------------------------------------------------ tcgen05
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// D[128 x N] (+)= A B with A and B in shared memory
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool acc)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc) : "memory");
}
// the same with A in TMEM
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool acc)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc) : "memory");
}
__device__ __forceinline__ void tc_ld32(uint32_t addr, float* v)
{
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
__device__ __forceinline__ void tc_st32(uint32_t addr, const float* v)
{
    const uint32_t* r = reinterpret_cast<const uint32_t*>(v);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
        ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
          "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
          "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t addr, const uint32_t* r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
        ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
// Shared-memory operand, 128-byte swizzle.  K-major (Q, K): rows of 128 bytes, groups of 8 rows `sbo` bytes apart.
// MN-major (V): 64 columns of a position are one 128-byte row, groups of 8 positions `sbo` apart, the next 64
// columns `lbo` away.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, uint32_t lbo, uint32_t sbo)
{
    return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(lbo >> 4) << 16) | ((uint64_t)(sbo >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}
constexpr uint32_t idesc_bf16(int n, bool b_mn_major)  // M = 128, fp32 accumulators
{
    return (1u << 4) | (1u << 7) | (1u << 10) | (b_mn_major ? 1u << 16 : 0u) | ((uint32_t)(n / 8) << 17) | ((128u / 16) << 24);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap* map, uint32_t bar, int slab, int head, int block, uint64_t policy)
{
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
        " [%0], [%1, {%2, %3, %4, %5, %6}], [%7], %8;"
        ::"r"(dst), "l"(map), "r"(0), "r"(0), "r"(slab), "r"(head), "r"(block), "r"(bar), "l"(policy)
        : "memory");
}
// bounded wait with one answer for the whole warp
__device__ __forceinline__ bool warp_wait(const uint64_t* bar, uint32_t parity, volatile int* abort_flag, int* status)
{
    return __all_sync(0xffffffffu, mbar_wait(smem_u32(bar), parity, abort_flag, status));
}

// ------------------------------------------------------------------ plan
// The same in every CTA, from the device-resident lengths, flags and groups.  CTA 0 also writes the descriptor that
// the second kernel works from, and reports what is wrong with the lengths and groups.
template <int TP>
__device__ __forceinline__ void shared_plan(const SharedParams& p, ShPlan& pl)
{
    const int tid = threadIdx.x, B = p.batch, NG = p.num_groups;
    const int cap = p.max_blocks_per_seq * kPage;
    int t_raw = 0, fl = 0;
    if (tid < B) {
        t_raw = p.seq_lens[tid];
        fl = p.flags[tid];
        pl.t[tid] = min(t_raw, cap);
        pl.act[tid] = fl && t_raw >= 1;
        if (fl && t_raw > cap && blockIdx.x == 0) atomicOr(p.status, kStatusBadSeqLen);
    }
    if (tid <= NG && NG > 0) pl.gs[tid] = p.group_start[tid];
    __syncthreads();
    if (tid < NG) {
        const int s = pl.gs[tid], e = pl.gs[tid + 1];
        bool ok = s >= 0 && e >= s && e <= B;
        for (int k = 0; k < tid; ++k) ok = ok && pl.gs[k] <= s;  // nobody belongs to two groups
        int n = 0, least = 0x7fffffff;
        if (ok) {
            for (int b = s; b < e; ++b)
                if (pl.act[b]) {
                    pl.list[s + n++] = (uint8_t)b;
                    least = min(least, pl.t[b]);
                }
        } else if (blockIdx.x == 0) {
            atomicOr(p.status, kStatusBadGroup);
        }
        // a lone request shares with nobody: its whole history is the second kernel's
        const int shared = n >= 2 ? min(p.group_prefix[tid], least - 1) : 0;
        pl.pages[tid] = shared > 0 ? shared / kPage : 0;
        pl.members[tid] = (uint8_t)n;
    }
    __syncthreads();
    if (tid < 32) {
        long long carry = 0;
        for (int i0 = 0; i0 < NG; i0 += 32) {
            const int i = i0 + tid;
            long long own = 0;
            if (i < NG) own = (long long)((pl.members[i] * p.group + 255) / 256) * ((pl.pages[i] + TP - 1) / TP);
            long long x = own;
            for (int o = 1; o < 32; o <<= 1) {
                const long long y = __shfl_up_sync(0xffffffffu, x, o);
                if (tid >= o) x += y;
            }
            if (i < NG) pl.off[i] = (int32_t)min(carry + x - own, 0x7fffffffll);
            carry += __shfl_sync(0xffffffffu, x, 31);
        }
        if (tid == 0) {
            long long total = carry * p.num_kv_heads * p.num_gated;
            if (carry > 0x7fffffffll || total > 0x7fffffffll) {  // beyond a 32-bit axis: nothing is shared
                if (blockIdx.x == 0) atomicOr(p.status, kStatusItemOverflow);
                total = carry = 0;
            }
            pl.off[NG] = (int32_t)carry;
            pl.t1 = (int32_t)carry;
            pl.total = (int32_t)total;
            pl.nseg = total > 0 ? (int)max(1ll, min((long long)gridDim.x, total / kShMinTiles)) : 0;
        }
    }
    __syncthreads();
    if (blockIdx.x == 0) {
        SharedDesc& d = *p.desc;
        if (tid == 0) {
            d.t1 = pl.t1;
            d.total = pl.total;
            d.nseg = pl.nseg;
        }
        for (int l = tid; l < p.num_gated; l += kShThreads) d.gated_index[p.layer[l]] = l;
        if (tid < B) {
            SharedRow r;
            r.unit = r.tiles = r.row = 0;
            int shift = 0;
            if (pl.total > 0 && pl.act[tid]) {
                for (int i = 0; i < NG; ++i) {
                    if (pl.pages[i] == 0 || tid < pl.gs[i] || tid >= pl.gs[i + 1]) continue;
                    int rank = 0;
                    for (int k = 0; k < pl.members[i]; ++k) rank += pl.list[pl.gs[i] + k] < tid;
                    const int per = 256 / p.group, block = rank / per;
                    r.tiles = (pl.pages[i] + TP - 1) / TP;
                    r.unit = pl.off[i] + block * r.tiles;
                    r.row = (rank - block * per) * p.group;
                    shift = pl.pages[i];
                }
            }
            d.rows[tid] = r;
            p.page_shift[tid] = shift;
            // what the second kernel sees of the request (a length below 1 is left for it to report)
            p.tail_lens[tid] = (t_raw < 1 ? t_raw : pl.t[tid]) - shift * kPage;
        }
    }
}

template <int TP>
__device__ __forceinline__ ShItem shared_item(const SharedParams& p, const ShPlan& pl, int x, int x_end)
{
    const int u = x / pl.t1, r = x - u * pl.t1;
    int lo = 0, hi = p.num_groups;  // last group that begins at or before r
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (pl.off[mid] <= r) lo = mid; else hi = mid;
    }
    ShItem it;
    it.gl = u / p.num_kv_heads;
    it.kvh = u - it.gl * p.num_kv_heads;
    it.group = lo;
    it.pages = pl.pages[lo];
    const int nt = (it.pages + TP - 1) / TP, r2 = r - pl.off[lo];
    const int block = r2 / nt;
    it.tile0 = r2 - block * nt;
    it.n = min(nt - it.tile0, x_end - x);
    it.row0 = block * 256;
    it.nrows = min(256, pl.members[lo] * p.group - it.row0);
    return it;
}

template <int D, int kTerms>
__global__ void __launch_bounds__(kShThreads, 1)
shared_prefix_kernel(const __grid_constant__ SharedParams p, const __grid_constant__ CUtensorMap kmap,
                     const __grid_constant__ CUtensorMap vmap)
{
    using C = ShCfg<D, kTerms>;
    constexpr int TP = C::kTilePages, TN = C::kTokens, kSlabs = D / 64;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* qs = smem;
    uint8_t* ring = smem + 2 * C::kQBytes;
    ShPlan& pl = *reinterpret_cast<ShPlan*>(ring + C::kSlots * C::kSlotBytes);
    ShCtl& ctl = *reinterpret_cast<ShCtl*>(reinterpret_cast<uint8_t*>(&pl) + (sizeof(ShPlan) + 15) / 16 * 16);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int* abort_flag = &ctl.abort;
    if (tid == 0) {
        for (int s = 0; s < C::kSlots; ++s) {
            mbar_init(smem_u32(&ctl.full[s]), 1);
            mbar_init(smem_u32(&ctl.empty[s]), 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(smem_u32(&ctl.s_full[s]), 1);
            mbar_init(smem_u32(&ctl.p_full[s]), 4);
            mbar_init(smem_u32(&ctl.o_full[s]), 1);
            mbar_init(smem_u32(&ctl.q_full[s]), 4);
        }
        mbar_init(smem_u32(&ctl.ml_full), 4);
        mbar_init(smem_u32(&ctl.o1_read), 4);
        ctl.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&kmap)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&vmap)) : "memory");
    }
    griddep_wait();
    shared_plan<TP>(p, pl);  // begins and ends its phases with barriers
    griddep_launch_dependents();
    const int span = (int)blockIdx.x;
    if (span >= pl.nseg) return;
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&ctl.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        tc_fence_before();
    }
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctl.tmem;
    const int x0 = (int)((long long)span * pl.total / pl.nseg), x1 = (int)((long long)(span + 1) * pl.total / pl.nseg);

    if (warp == 8) {
        // ============================ producer warp ============================
        const uint64_t once = 0x12F0000000000000ull;    // L2 evict-first: read by one row block
        const uint64_t again = 0x1000000000000000ull;   // L2 evict-normal: the next row block reads it too
        uint32_t cnt = 0;
        bool dead = false;
        for (int x = x0; x < x1 && !dead;) {
            const ShItem it = shared_item<TP>(p, pl, x, x1);
            x += it.n;
            const int ahead = it.nrows > kShRows ? 1 : 2;
            const int lead = pl.list[pl.gs[it.group]];
            const int32_t* table = p.block_table + (size_t)lead * p.max_blocks_per_seq;
            const int first = it.tile0 * TP, last = min(it.pages, (it.tile0 + it.n) * TP);
            const int kv0 = p.kv_index[it.gl] * p.blocks_per_layer;
            const uint64_t policy = pl.members[it.group] * p.group > 256 ? again : once;
            // block ids of 32 pages from page `base` on, the lanes' own; K runs up to two tiles ahead of V
            int base_k = -64, ids_k = 0, base_v = -64, ids_v = 0;
            auto load = [&](int tile, bool is_v) {
                const int pg = first + tile * TP, np = min(TP, last - pg);
                int& base = is_v ? base_v : base_k;
                int& ids = is_v ? ids_v : ids_k;
                if (pg - base >= 32) {
                    base = pg;
                    ids = pg + lane < last ? __ldg(table + pg + lane) : 0;
                }
                const uint32_t s = cnt % C::kSlots, ph = (cnt / C::kSlots) & 1;
                if (!warp_wait(&ctl.empty[s], ph ^ 1, abort_flag, p.status)) return false;
                const uint32_t bar = smem_u32(&ctl.full[s]);
                if (lane == 0) mbar_expect_tx(bar, (uint32_t)np * kPage * D * 2);
                __syncwarp();
                const uint32_t dst = smem_u32(ring + s * C::kSlotBytes);
                if (is_v) {  // one box: the page of the head, slab after slab
                    const int blk = __shfl_sync(0xffffffffu, ids, (pg - base + (lane & (TP - 1))) & 31);
                    if (lane < np) tma_box(dst + lane * (kPage * D * 2), &vmap, bar, 0, it.kvh, kv0 + blk, policy);
                } else {     // one box per slab: a slab's rows of all pages lie one behind the other
                    const int pgi = lane % TP, slab = lane / TP;
                    const int blk = __shfl_sync(0xffffffffu, ids, (pg - base + pgi) & 31);
                    if (pgi < np && slab < kSlabs) tma_box(dst + slab * (TN * 128) + pgi * 2048, &kmap, bar, slab, it.kvh, kv0 + blk, policy);
                }
                ++cnt;
                return true;
            };
            bool ok = true;
            for (int t = 0; t < min(ahead, it.n) && ok; ++t) ok = load(t, false);
            for (int t = 0; t < it.n && ok; ++t) {
                ok = load(t, true);
                if (ok && t + ahead < it.n) ok = load(t + ahead, false);
            }
            dead = !ok;
        }
        // do not leave while copies may still be landing: every armed slot has been released (bounded)
        for (uint32_t k = 0; k < (uint32_t)C::kSlots && k < cnt; ++k) {
            const uint32_t c2 = cnt - 1 - k;
            if (!warp_wait(&ctl.empty[c2 % C::kSlots], (c2 / C::kSlots) & 1, abort_flag, p.status)) break;
        }
    } else if (warp == 9) {
        // ============================ MMA warp (one thread) ============================
        if (lane == 0) {
            constexpr uint32_t idesc_s = idesc_bf16(TN, false), idesc_o = idesc_bf16(D, true);
            uint32_t cnt = 0, nq[2] = {0, 0}, np_[2] = {0, 0};
            bool ok = true;
            auto acquire = [&]() {  // next slot of the ring, in the producer's order
                const uint32_t s = cnt % C::kSlots, ph = (cnt / C::kSlots) & 1;
                ++cnt;
                ok = mbar_wait(smem_u32(&ctl.full[s]), ph, abort_flag, p.status);
                tc_fence_after();
                return s;
            };
            auto qk = [&](int s, uint32_t slot) {  // S of stream s, whole tile (columns past the last page are not used)
                const uint32_t a = smem_u32(qs + s * C::kQBytes), b = smem_u32(ring + slot * C::kSlotBytes);
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    tc_mma_ss(tmem + s * C::kSpCols, smem_desc(a + (k >> 2) * (kShRows * 128) + (k & 3) * 32, 16, 1024),
                              smem_desc(b + (k >> 2) * (TN * 128) + (k & 3) * 32, 16, 1024), idesc_s, k > 0);
                tc_commit(smem_u32(&ctl.s_full[s]));
            };
            auto pv = [&](int s, uint32_t slot, int pages, bool first) {
                ok = mbar_wait(smem_u32(&ctl.p_full[s]), np_[s]++ & 1, abort_flag, p.status);
                if (!ok) return;
                tc_fence_after();
                const uint32_t b = smem_u32(ring + slot * C::kSlotBytes);
                for (int k = 0; k < pages; ++k) {  // a page is one K step of 16 positions
                    const uint64_t bd = smem_desc(b + k * (kPage * D * 2), 2048, 1024);
#pragma unroll
                    for (int c = 0; c < kTerms; ++c)
                        tc_mma_ts(tmem + C::kO0 + s * D, tmem + s * C::kSpCols + c * (TN / 2) + k * 8, bd, idesc_o,
                                  !first || k > 0 || c > 0);
                }
            };
            auto wait_q = [&](int s) {
                ok = mbar_wait(smem_u32(&ctl.q_full[s]), nq[s]++ & 1, abort_flag, p.status);
                tc_fence_after();
            };
            for (int x = x0; x < x1 && ok;) {
                const ShItem it = shared_item<TP>(p, pl, x, x1);
                x += it.n;
                const int first = it.tile0 * TP;
                auto pages_of = [&](int t) { return min(TP, it.pages - first - t * TP); };
                if (it.nrows > kShRows) {
                    wait_q(0);
                    if (ok) wait_q(1);
                    uint32_t ks = ok ? acquire() : 0;
                    if (!ok) break;
                    qk(0, ks);
                    qk(1, ks);
                    tc_commit(smem_u32(&ctl.empty[ks]));
                    for (int t = 0; t < it.n; ++t) {
                        const uint32_t vs = acquire();
                        if (!ok) break;
                        const bool more = t + 1 < it.n;
                        pv(0, vs, pages_of(t), t == 0);
                        if (!ok) break;
                        if (more) {
                            ks = acquire();
                            if (!ok) break;
                            qk(0, ks);
                        } else {
                            tc_commit(smem_u32(&ctl.o_full[0]));
                        }
                        pv(1, vs, pages_of(t), t == 0);
                        if (!ok) break;
                        tc_commit(smem_u32(&ctl.empty[vs]));
                        if (more) {
                            qk(1, ks);
                            tc_commit(smem_u32(&ctl.empty[ks]));
                        } else {
                            tc_commit(smem_u32(&ctl.o_full[1]));
                        }
                    }
                } else {
                    for (int t = 0; t < min(2, it.n) && ok; ++t) {
                        wait_q(t);
                        const uint32_t ks = ok ? acquire() : 0;
                        if (!ok) break;
                        qk(t, ks);
                        tc_commit(smem_u32(&ctl.empty[ks]));
                    }
                    for (int t = 0; t < it.n && ok; ++t) {
                        const int s = t & 1;
                        const uint32_t vs = acquire();
                        if (!ok) break;
                        pv(s, vs, pages_of(t), t < 2);
                        if (!ok) break;
                        tc_commit(smem_u32(&ctl.empty[vs]));
                        if (t + 2 < it.n) {
                            const uint32_t ks = acquire();
                            if (!ok) break;
                            qk(s, ks);
                            tc_commit(smem_u32(&ctl.empty[ks]));
                        } else {
                            tc_commit(smem_u32(&ctl.o_full[s]));
                        }
                    }
                }
            }
        }
        __syncwarp();
    } else {
        // ============================ softmax warpgroups: one thread per row ============================
        const int s = warp >> 2;                     // stream
        const int tr = tid & (kShRows - 1);          // row of the tile = TMEM lane
        const uint32_t sp = tmem + ((uint32_t)(warp & 3) << 21) + s * C::kSpCols;
        const uint32_t oc = tmem + ((uint32_t)(warp & 3) << 21) + C::kO0;
        const float scale = p.scale_log2e;
        uint32_t ns = 0, no = 0, nj = 0;
        bool ok = true;
        for (int x = x0; x < x1 && ok;) {
            const ShItem it = shared_item<TP>(p, pl, x, x1);
            x += it.n;
            const bool dual = it.nrows > kShRows;
            if (!dual && s == 1 && it.n == 1) continue;  // a lone tile: stream 0's
            const int row = dual ? s * kShRows + tr : tr;
            const bool valid = row < it.nrows;
            const bool warp_valid = (row & ~31) < it.nrows;
            const int layer = p.layer[it.gl];
            int b = 0, head = 0;
            if (valid) {
                const int r = it.row0 + row;
                b = pl.list[pl.gs[it.group] + r / p.group];
                head = it.kvh * p.group + r % p.group;
                const uint4* src = reinterpret_cast<const uint4*>(p.q + (((size_t)layer * p.batch + b) * p.num_q_heads + head) * D);
                uint8_t* dst = qs + s * C::kQBytes + tr * 128;
                uint4 v[D / 8];
#pragma unroll
                for (int c = 0; c < D / 8; ++c) v[c] = __ldg(src + c);
#pragma unroll
                for (int c = 0; c < D / 8; ++c)
                    *reinterpret_cast<uint4*>(dst + (c >> 3) * (kShRows * 128) + (((c & 7) ^ (tr & 7)) << 4)) = v[c];
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctl.q_full[s]));
            float m = -INFINITY, l = 0.f;  // m in log2 units
            bool fresh = true;
            for (int t = dual ? 0 : s; t < it.n; t += dual ? 1 : 2) {
                if (!warp_wait(&ctl.s_full[s], ns++ & 1, abort_flag, p.status)) { ok = false; break; }
                tc_fence_after();
                if (warp_valid) {
                    const int cols = min(TP, it.pages - (it.tile0 + t) * TP) * kPage;
                    float v[TN];
#pragma unroll
                    for (int c = 0; c < TN; c += 32) tc_ld32(sp + c, v + c);
                    tc_wait_ld();
                    if (cols < TN) {
#pragma unroll
                        for (int c = 0; c < TN; ++c) v[c] = c < cols ? v[c] : -INFINITY;
                    }
                    float mx[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
                    for (int c = 4; c < TN; ++c) mx[c & 3] = fmaxf(mx[c & 3], v[c]);
                    const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale;
                    // The running maximum only moves when it would grow by more than 2^8: any value near the true one
                    // gives the same quotient, and O in TMEM then rarely has to be scaled.
                    if (fresh) {
                        m = top;
                        fresh = false;
                    } else if (__any_sync(0xffffffffu, top > m + 8.f)) {
                        // S of this tile is complete, so the products of the tiles before it are too: O is at rest
                        const float mn = top > m + 8.f ? top : m;
                        const float a = m == -INFINITY ? 0.f : ex2(m - mn);
                        m = mn;
                        l *= a;
#pragma unroll
                        for (int c = 0; c < D; c += 32) {
                            float o[32];
                            tc_ld32(oc + s * D + c, o);
                            tc_wait_ld();
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] *= a;
                            tc_st32(oc + s * D + c, o);
                        }
                    }
                    const float mu = m == -INFINITY ? 0.f : m;
                    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c0 = 0; c0 < TN; c0 += 32) {
                        uint32_t part[kTerms][16];
#pragma unroll
                        for (int e = 0; e < 32; e += 2) {
                            float a = ex2(fmaf(v[c0 + e], scale, -mu)), c = ex2(fmaf(v[c0 + e + 1], scale, -mu));
                            sum[e & 3] += a;
                            sum[(e + 1) & 3] += c;
#pragma unroll
                            for (int k = 0; k < kTerms; ++k) {
                                const uint32_t pk = pack2(a, c);
                                part[k][e / 2] = pk;
                                a -= __uint_as_float(pk << 16);
                                c -= __uint_as_float(pk & 0xffff0000u);
                            }
                        }
#pragma unroll
                        for (int k = 0; k < kTerms; ++k) tc_st16(sp + k * (TN / 2) + c0 / 2, part[k]);
                    }
                    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                    tc_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&ctl.p_full[s]));
            }
            if (!ok) break;
            if (!warp_wait(&ctl.o_full[s], no++ & 1, abort_flag, p.status)) { ok = false; break; }
            tc_fence_after();
            // ---- the item's partial: chunk 0 of a unit in the row's own place, later chunks in the span's ----
            const bool joined = !dual && it.n > 1;
            float a0 = 1.f, a1 = 0.f;
            if (joined) {
                if (s == 1) {
                    ctl.ml1[tr] = make_float2(m, l);
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&ctl.ml_full));
                } else {
                    if (!warp_wait(&ctl.ml_full, nj & 1, abort_flag, p.status)) { ok = false; break; }
                    tc_fence_after();
                    const float2 o = ctl.ml1[tr];
                    const float mn = fmaxf(m, o.x), mu = mn == -INFINITY ? 0.f : mn;
                    a0 = ex2(m - mu);
                    a1 = ex2(o.x - mu);
                    m = mn;
                    l = l * a0 + o.y * a1;
                }
            }
            if (warp_valid && (dual || s == 0)) {
                const size_t dst = it.tile0 == 0 ? ((size_t)it.gl * p.batch + b) * p.num_q_heads + head
                                                 : p.ext_row0 + (size_t)span * 256 + row;
#pragma unroll
                for (int c = 0; c < D; c += 32) {
                    float o[32];
                    tc_ld32(oc + s * D + c, o);
                    if (joined) {
                        float o1[32];
                        tc_ld32(oc + D + c, o1);
                        tc_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = o[e] * a0 + o1[e] * a1;
                    } else {
                        tc_wait_ld();
                    }
                    if (valid) {
                        float4* to = reinterpret_cast<float4*>(p.part_o + dst * D + c);
#pragma unroll
                        for (int e = 0; e < 32; e += 4) __stcg(to + e / 4, make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]));
                    }
                }
                if (valid) __stcg(p.part_ml + dst, make_float2(m, l));
            }
            tc_fence_before();
            if (joined) {  // stream 1's next item may overwrite its O and (m, l) once stream 0 has read them
                __syncwarp();
                if (s == 0) {
                    if (lane == 0) mbar_arrive(smem_u32(&ctl.o1_read));
                } else if (!warp_wait(&ctl.o1_read, nj & 1, abort_flag, p.status)) {
                    ok = false;
                    break;
                }
                ++nj;
            }
        }
    }
    // Every wait above is bounded, so all warps come here; after an abandoned wait, copies and products in flight get
    // time to land before shared memory and TMEM are given back.
    if (*abort_flag)
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

template <int D, int kTerms>
static cudaError_t launch_shared_t(const SharedParams& p, const void* kmap, const void* vmap, int grid, cudaStream_t st, bool pdl)
{
    using C = ShCfg<D, kTerms>;
    constexpr int smem = 2 * C::kQBytes + C::kSlots * C::kSlotBytes + (int)(sizeof(ShPlan) + 15) / 16 * 16 + (int)sizeof(ShCtl);
    static_assert(smem <= 232448, "shared memory");
    cudaError_t e = cudaFuncSetAttribute(shared_prefix_kernel<D, kTerms>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    return launch_ex(shared_prefix_kernel<D, kTerms>, dim3(grid), dim3(kShThreads), smem, st, pdl, p,
                     *reinterpret_cast<const CUtensorMap*>(kmap), *reinterpret_cast<const CUtensorMap*>(vmap));
}

cudaError_t launch_shared_prefix(const SharedParams& p, const void* kmap, const void* vmap, int head_dim, bool out_bf16,
                                 int grid, cudaStream_t st, bool pdl)
{
    if (head_dim == 128)
        return out_bf16 ? launch_shared_t<128, 2>(p, kmap, vmap, grid, st, pdl) : launch_shared_t<128, 3>(p, kmap, vmap, grid, st, pdl);
    return out_bf16 ? launch_shared_t<64, 2>(p, kmap, vmap, grid, st, pdl) : launch_shared_t<64, 3>(p, kmap, vmap, grid, st, pdl);
}

}  // namespace oda
