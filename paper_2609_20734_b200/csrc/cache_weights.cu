// Accumulated attention weights: the second kernel of the weighted Full pass.
//
//   W[slice, b, g, j] += sum over the group's heads h of 2^(x_hj - m_h) / l_h
//
// x are the logits (log2 units) that the attention kernel left, (m, 1 / l) the finished softmax of each row.
// The weights of a row are only known once its last page has been seen, so they cannot be added up inside the
// pass; writing the logits (4 bytes a head and position) and reading them back costs 8 G of the 4 D bytes a
// position that reading K a second time would half repeat.  Memory bound: 4 G + 8 bytes a position (32 layers of 8 heads,
// 32,768 positions, G = 4: 201 MB, 30 us behind the pass's 673, 6.7 TB/s: the last logits come from L2).
//
// A position is added by one thread, heads in index order and layers that share a cache slice in layer order:
// no atomics, the same bits every time.
#include "launch_ex.cuh"
#include "oda_device.cuh"
#include "oda_launch.h"

namespace oda {

constexpr int kAccThreads = 256;
constexpr int kAccPerThread = 4;

template <int G>
__global__ void __launch_bounds__(kAccThreads)
accumulate_weights_kernel(const __grid_constant__ WeightParams p)
{
    griddep_wait();
    griddep_launch_dependents();
    const uint32_t unit = blockIdx.x / p.chunks, chunk = blockIdx.x - unit * p.chunks;  // (x: units may be more than 65,535)
    const int b = unit / p.num_kv_heads, g = unit - b * p.num_kv_heads;
    if (!p.flags[b]) return;
    const size_t max_pos = (size_t)p.max_blocks_per_seq * kPage;
    const int t = (int)min((long long)p.seq_lens[b], (long long)max_pos);  // the attention kernel reports what is beyond
    const int j0 = (int)chunk * (kAccThreads * kAccPerThread) + threadIdx.x;
    if (j0 >= t) return;
    const int first = p.first_layer[blockIdx.y];  // of the call's gated layers that use this slice
    float* w = p.weights + (((size_t)p.slice[blockIdx.y] * p.max_batch + b) * p.num_kv_heads + g) * max_pos;
    float acc[kAccPerThread];
#pragma unroll
    for (int i = 0; i < kAccPerThread; ++i) acc[i] = j0 + i * kAccThreads < t ? w[j0 + i * kAccThreads] : 0.f;
    for (int l = first; l >= 0; l = p.next_layer[l]) {
        const float2* ml = p.score_ml + ((size_t)l * p.batch + b) * (p.num_kv_heads * G) + g * G;
        float2 r[G];
#pragma unroll
        for (int h = 0; h < G; ++h) r[h] = ml[h];
        const float* x = p.score_rows + (((size_t)l * p.batch + b) * p.num_kv_heads + g) * max_pos * G;
        float v[kAccPerThread][G];
#pragma unroll
        for (int i = 0; i < kAccPerThread; ++i) {
            const int j = min(j0 + i * kAccThreads, t - 1);
            if constexpr (G >= 4) {
#pragma unroll
                for (int h = 0; h < G; h += 4) {
                    const float4 q = __ldcs(reinterpret_cast<const float4*>(x + (size_t)j * G + h));
                    v[i][h] = q.x; v[i][h + 1] = q.y; v[i][h + 2] = q.z; v[i][h + 3] = q.w;
                }
            } else if constexpr (G == 2) {
                const float2 q = __ldcs(reinterpret_cast<const float2*>(x + (size_t)j * G));
                v[i][0] = q.x; v[i][1] = q.y;
            } else {
                v[i][0] = __ldcs(x + j);
            }
        }
#pragma unroll
        for (int i = 0; i < kAccPerThread; ++i) {
            float s = 0.f;
#pragma unroll
            for (int h = 0; h < G; ++h) s = fmaf(ex2(v[i][h] - r[h].x), r[h].y, s);
            acc[i] += s;
        }
    }
#pragma unroll
    for (int i = 0; i < kAccPerThread; ++i)
        if (j0 + i * kAccThreads < t) w[j0 + i * kAccThreads] = acc[i];
}

cudaError_t launch_accumulate_weights(const WeightParams& args, int n_slices, int group, cudaStream_t st, bool pdl)
{
    const long long max_pos = (long long)args.max_blocks_per_seq * kPage;
    const int per = kAccThreads * kAccPerThread;
    WeightParams p = args;
    p.chunks = (int32_t)((max_pos + per - 1) / per);
    const long long x = (long long)p.chunks * p.batch * p.num_kv_heads;
    if (x > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    const dim3 grid((unsigned)x, n_slices);
    switch (group) {
        case 1: return launch_ex(accumulate_weights_kernel<1>, grid, dim3(kAccThreads), 0, st, pdl, p);
        case 2: return launch_ex(accumulate_weights_kernel<2>, grid, dim3(kAccThreads), 0, st, pdl, p);
        case 4: return launch_ex(accumulate_weights_kernel<4>, grid, dim3(kAccThreads), 0, st, pdl, p);
        default: return launch_ex(accumulate_weights_kernel<8>, grid, dim3(kAccThreads), 0, st, pdl, p);
    }
}

}  // namespace oda
