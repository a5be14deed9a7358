// Eviction of a paged cache down to a budget, by accumulated attention weight.
//
// For every (cache slice, request, kv head) with t > budget positions, the kept set is
//   {0 .. sinks-1}  u  {t-recent .. t-1}  u  the (budget - sinks - recent) heaviest positions between them
// (ties to the lowest index); K, V and the weights of the kept positions move to 0 .. budget-1 in order of position.
//
// 1. evict_select_kernel finds the kept set: a radix select over the order-preserving 32-bit image of the weights (four
//    8-bit digits, most significant first) gives the lightest kept weight T and how many positions of exactly T
//    belong to the set; one ordered pass with a prefix sum writes the list of kept positions and compacts the weights.
// 2. evict_move_kernel moves the rows in place.  Destination i never lies behind its source (i <= kept[i], both
//    rising), so a chunk of rows whose sources have all been read may be written: later sources lie behind it.
#include "launch_ex.cuh"
#include "oda_device.cuh"
#include "oda_launch.h"

namespace oda {

constexpr int kSelThreads = 1024;
constexpr int kMoveThreads = 512;
constexpr int kMovePieces = 8;  // 16-byte pieces a thread holds of one chunk

// larger weight -> larger key; -0 and +0 are one key, NaN is above everything
__device__ __forceinline__ uint32_t weight_key(float w)
{
    const uint32_t u = __float_as_uint(w + 0.f);  // -0 + 0 = +0
    if (w != w) return 0xffffffffu;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__global__ void __launch_bounds__(kSelThreads)
evict_select_kernel(const __grid_constant__ EvictParams p)
{
    griddep_wait();
    griddep_launch_dependents();
    __shared__ uint32_t hist[256];
    __shared__ uint32_t s_prefix, s_left;
    __shared__ uint32_t wsum[kSelThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int unit = blockIdx.x;  // (slice, request, head)
    const int g = unit % p.num_kv_heads, b = (unit / p.num_kv_heads) % p.batch, slice = unit / (p.num_kv_heads * p.batch);
    if (p.mask && !p.mask[b]) return;
    const int t = p.seq_lens[b];
    const size_t max_pos = (size_t)p.max_blocks_per_seq * kPage;
    if (t < 1 || (size_t)t > max_pos) {
        if (tid == 0) atomicOr(p.status, kStatusBadSeqLen);
        return;
    }
    int32_t* kept = p.kept + (size_t)unit * p.budget;
    const int n = p.budget;
    if (t <= n) {  // nothing to drop
        for (int i = tid; i < n; i += kSelThreads) kept[i] = i < t ? i : -1;
        return;
    }
    float* w = p.weights + (((size_t)slice * p.max_batch + b) * p.num_kv_heads + g) * max_pos;
    const int lo = p.sinks, hi = t - p.recent;  // candidates
    uint32_t left = (uint32_t)(n - p.sinks - p.recent);  // how many of them stay (less than hi - lo)
    uint32_t prefix = 0;
    if (left > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < 256; i += kSelThreads) hist[i] = 0;
            __syncthreads();
            const uint32_t above = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
            for (int i = lo + tid; i < hi; i += kSelThreads) {
                const uint32_t k = weight_key(w[i]);
                if ((k & above) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
            }
            __syncthreads();
            if (warp == 0) {  // the digit in which the count from above reaches `left`
                uint32_t c[8], sum = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) { c[k] = hist[255 - (lane * 8 + k)]; sum += c[k]; }
                uint32_t x = sum;
                for (int o = 1; o < 32; o <<= 1) {
                    const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
                    if (lane >= o) x += y;
                }
                uint32_t before = x - sum;
                if (before < left && x >= left) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (before < left && before + c[k] >= left) {
                            s_prefix = prefix | ((uint32_t)(255 - (lane * 8 + k)) << shift);
                            s_left = left - before;
                            break;
                        }
                        before += c[k];
                    }
                }
            }
            __syncthreads();
            prefix = s_prefix;
            left = s_left;
        }
    }
    // ordered pass: heavier than T, or T itself while `left` of them last
    const uint32_t T = prefix;
    const bool any = n > p.sinks + p.recent;
    uint32_t base_gt = 0, base_eq = 0;
    for (int i0 = 0; i0 < t; i0 += kSelThreads) {
        const int i = i0 + tid;
        float val = 0.f;
        uint32_t gt = 0, eq = 0;
        if (i < t) {
            val = w[i];
            const uint32_t k = weight_key(val);
            const bool fixed = i < lo || i >= hi;
            gt = fixed || (any && k > T);
            eq = !fixed && any && k == T;
        }
        uint32_t x = gt | (eq << 16);  // at most 1024 of each in a block
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) wsum[warp] = x;
        __syncthreads();
        if (warp == 0) {
            uint32_t y = wsum[lane];
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t z = __shfl_up_sync(0xffffffffu, y, o);
                if (lane >= o) y += z;
            }
            wsum[lane] = y;
        }
        __syncthreads();
        const uint32_t incl = x + (warp ? wsum[warp - 1] : 0);
        const uint32_t gts = base_gt + (incl & 0xffffu) - gt, eqs = base_eq + (incl >> 16) - eq;
        if (gt || (eq && eqs < left)) {
            const uint32_t dst = gts + min(eqs, left);
            kept[dst] = i;
            w[dst] = val;  // dst <= i, and every weight up to this block's end has been read
        }
        base_gt += wsum[31] & 0xffffu;
        base_eq += wsum[31] >> 16;
        __syncthreads();
    }
    for (int i = n + tid; i < t; i += kSelThreads) w[i] = 0.f;
}

template <int D>
__global__ void __launch_bounds__(kMoveThreads)
evict_move_kernel(const __grid_constant__ EvictParams p)
{
    griddep_wait();
    griddep_launch_dependents();
    constexpr int kRowPieces = D / 8;                                  // 16-byte pieces of one K (or V) row
    constexpr int kRows = kMoveThreads * kMovePieces / (2 * kRowPieces);  // rows of one chunk, K and V
    const int tid = threadIdx.x;
    const int unit = blockIdx.x;
    const int g = unit % p.num_kv_heads, b = (unit / p.num_kv_heads) % p.batch, slice = unit / (p.num_kv_heads * p.batch);
    const int t = p.seq_lens[b];
    const int n = p.budget;
    const bool work = (!p.mask || p.mask[b]) && t > n && (size_t)t <= (size_t)p.max_blocks_per_seq * kPage;
    if (work) {
        const int32_t* kept = p.kept + (size_t)unit * n;
        // kept[i] - i never falls: the rows that stay where they are come first
        int i0 = 0, i1 = n;
        while (i0 < i1) {
            const int mid = (i0 + i1) >> 1;
            if (kept[mid] == mid) i0 = mid + 1; else i1 = mid;
        }
        const int32_t* table = p.block_table + (size_t)b * p.max_blocks_per_seq;
        const size_t unit_off = (size_t)slice * p.kv_layer_stride + (size_t)g * p.kv_head_stride;
        auto row = [&](int pos) {
            return unit_off + (size_t)table[pos / kPage] * p.kv_block_stride + (size_t)(pos % kPage) * p.kv_token_stride;
        };
        for (; i0 < n; i0 += kRows) {
            uint4 x[kMovePieces];
#pragma unroll
            for (int k = 0; k < kMovePieces; ++k) {
                const int e = tid + k * kMoveThreads;
                const int r = e / (2 * kRowPieces), c = e % (2 * kRowPieces);
                if (i0 + r < n) {
                    const __nv_bfloat16* base = c < kRowPieces ? p.k : p.v;
                    x[k] = *reinterpret_cast<const uint4*>(base + row(kept[i0 + r]) + (size_t)(c % kRowPieces) * 8);
                }
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kMovePieces; ++k) {
                const int e = tid + k * kMoveThreads;
                const int r = e / (2 * kRowPieces), c = e % (2 * kRowPieces);
                if (i0 + r < n) {
                    __nv_bfloat16* base = c < kRowPieces ? p.k : p.v;
                    *reinterpret_cast<uint4*>(base + row(i0 + r) + (size_t)(c % kRowPieces) * 8) = x[k];
                }
            }
            __syncthreads();
        }
    }
    // the CTA that comes last shortens the requests: nobody reads their lengths any more
    if (tid == 0) {
        __threadfence();
        if (atomicAdd(p.done, 1) == (int)gridDim.x - 1) {
            *p.done = 0;
            for (int r = 0; r < p.batch; ++r)
                if ((!p.mask || p.mask[r]) && p.seq_lens[r] > n && (size_t)p.seq_lens[r] <= (size_t)p.max_blocks_per_seq * kPage)
                    p.seq_lens[r] = n;
        }
    }
}

cudaError_t launch_evict(const EvictParams& p, int head_dim, cudaStream_t st, bool pdl)
{
    const unsigned units = (unsigned)(p.num_slices * p.batch * p.num_kv_heads);
    cudaError_t e = launch_ex(evict_select_kernel, dim3(units), dim3(kSelThreads), 0, st, pdl, p);
    if (e != cudaSuccess) return e;
    if (head_dim == 128) return launch_ex(evict_move_kernel<128>, dim3(units), dim3(kMoveThreads), 0, st, pdl, p);
    return launch_ex(evict_move_kernel<64>, dim3(units), dim3(kMoveThreads), 0, st, pdl, p);
}

}  // namespace oda
