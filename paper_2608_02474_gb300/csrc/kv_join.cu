// The second launch of an attention call over the paged cache: items that several CTAs did
// in pieces (kv_schedule.cuh) become outputs.
#include <cfloat>

#include "kv_schedule.cuh"

namespace {

// Blocks (c, .): the item that worker c began and others went on with, a warp per row.
// With the pieces' maxima m_i and sums l_i: out = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i,
// m = max_i m_i, in the order of the keys.
constexpr int kWarps = 8;

template <int D>
__global__ void __launch_bounds__(32 * kWarps)
kv_join_kernel(const KvWork w, float *ws, __nv_bfloat16 *__restrict__ out, int64_t ldo) {
    pdl_enter();
    const KvJoin j = kv_joins(ws, w, D)[blockIdx.x];
    if (j.more == 0) return;
    constexpr int E = D / 32;
    const int lane = threadIdx.x & 31, n = 1 + j.more;
    const int64_t slot = (int64_t)w.slot_rows * (D + 2);
    // piece 0 in this worker's second slot, piece i in worker c + i's first
    auto piece = [&](int i) -> const float * { return ws + slot * (2 * (blockIdx.x + i) + (i == 0 ? 1 : 0)); };
    for (int row = blockIdx.y * kWarps + ((int)threadIdx.x >> 5); row < j.rows; row += gridDim.y * kWarps) {
        float m = -FLT_MAX;
        for (int i = lane; i < n; i += 32) m = fmaxf(m, piece(i)[w.slot_rows * D + 2 * row]);
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
        float l = 0.f, acc[E] = {};
        for (int i0 = 0; i0 < n; i0 += 32) {
            float f = 0.f, li = 0.f;                                   // of piece i0 + lane
            if (i0 + lane < n) {
                const float2 ml = *reinterpret_cast<const float2 *>(piece(i0 + lane) + w.slot_rows * D + 2 * row);
                f = ex2_approx(ml.x - m);
                li = f * ml.y;
            }
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) li += __shfl_xor_sync(0xffffffffu, li, x);
            l += li;
            const int some = min(32, n - i0);
#pragma unroll 8
            for (int i = 0; i < some; ++i) {
                const float fi = __shfl_sync(0xffffffffu, f, i);
                const float *src = piece(i0 + i) + row * D + lane * E;
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const float2 v = *reinterpret_cast<const float2 *>(src + e);
                    acc[e] += fi * v.x;
                    acc[e + 1] += fi * v.y;
                }
            }
        }
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int pr = j.packed0 + row;
        __nv_bfloat16 *dst = out + (int64_t)(j.row + pr / w.group) * ldo +
                             (j.head * w.group + pr % w.group) * D + lane * E;
#pragma unroll
        for (int e = 0; e < E; e += 2)
            *reinterpret_cast<uint32_t *>(dst + e) = pack_bf16(acc[e] * inv, acc[e + 1] * inv);
    }
}

}  // namespace

namespace echo {

void launch_kv_join(const KvAttention &a, const KvWork &w, cudaStream_t st) {
    if (!w.split) return;
    const int d = a.pool->d;
    const int rows = w.tile / kWarps < 8 ? (w.tile + kWarps - 1) / kWarps : 8;
    LaunchScope ls(ECHO_K_KV_JOIN, a.batch->n_rows, (int64_t)a.Hq * d, w.workers, st);
    launch_chained(d == 64 ? kv_join_kernel<64> : kv_join_kernel<128>, dim3(w.workers, rows), dim3(32 * kWarps), 0,
                   st, w, static_cast<float *>(a.ws), static_cast<__nv_bfloat16 *>(a.out), a.ldo);
}

}  // namespace echo
