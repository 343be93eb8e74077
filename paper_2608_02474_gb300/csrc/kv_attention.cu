// Attention of new rows over the paged key/value cache: the plainest form, a warp per
// (row, query head) that walks the row's keys once with a running maximum and sum.
#include <cfloat>

#include "kv_pages.cuh"

namespace {

constexpr int kThreads = 128;

template <bool INT8, int D>
__global__ void __launch_bounds__(kThreads)
kv_attention_kernel(const KvPool pool, const KvBatch b, const __nv_bfloat16 *__restrict__ q, int64_t ldq,
                    int Hq, int causal_block, float scale_log2, __nv_bfloat16 *__restrict__ out,
                    int64_t ldo, int *err) {
    pdl_enter();
    constexpr int E = D / 32;                       // values of a lane
    const int lane = threadIdx.x & 31;
    for (PieceWalk walk(blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), gridDim.x * (kThreads / 32), Hq);
         walk.below(b.n_rows); walk.next()) {
        const int r = (int)walk.row, h = (int)walk.piece, g = h / (Hq / pool.H);
        const int seq = kv_seq_of_row(b, r);
        if (seq < 0) continue;
        const int64_t len = b.len[seq], p = len - b.row0[seq + 1] + r;
        int64_t top = len;
        if (causal_block > 0) top = p < 0 ? 0 : min(len, (p / causal_block + 1) * causal_block);
        float qv[E], o[E] = {}, m = -FLT_MAX, l = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) qv[e] = __bfloat162float(q[r * ldq + h * D + lane * E + e]) * scale_log2;
        for (int64_t j = 0; j < top; ++j) {
            const int64_t at = kv_place(pool, b, seq, j, err);
            if (at < 0) break;
            const int64_t page = at >> pool.shift, slot = at & ((1 << pool.shift) - 1);
            const int64_t kvec = (((page * 2) * pool.H + g) << pool.shift) + slot;
            const int64_t vvec = (((page * 2 + 1) * pool.H + g) << pool.shift) + slot;
            auto value = [&](int64_t vec, int e) -> float {
                if constexpr (INT8) return (float)reinterpret_cast<const int8_t *>(pool.pages)[vec * D + lane * E + e];
                else return __bfloat162float(reinterpret_cast<const __nv_bfloat16 *>(pool.pages)[vec * D + lane * E + e]);
            };
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) s += qv[e] * value(kvec, e);
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
            float w = 1.f;
            if constexpr (INT8) { s *= pool.scale[kvec]; w = pool.scale[vvec]; }
            const float m2 = fmaxf(m, s), a = ex2_approx(m - m2), pr = ex2_approx(s - m2);
            m = m2;
            l = l * a + pr;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = o[e] * a + pr * w * value(vvec, e);
        }
        const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;   // no keys: 0; NaN stays
#pragma unroll
        for (int e = 0; e < E; ++e) out[r * ldo + h * D + lane * E + e] = __float2bfloat16_rn(o[e] * inv);
    }
}

}  // namespace

extern "C" size_t echo_kv_attention_workspace_size(const echo_kv_pool *pool, const echo_kv_batch *batch,
                                                   int32_t Hq) {
    bool empty;
    if (Hq < 1 || echo::kv_check(pool, batch, &empty) != ECHO_OK) return 0;
    return 256;
}

extern "C" echo_status echo_kv_attention(const echo_kv_pool *pool, const echo_kv_batch *batch,
                                         const void *q, int64_t ldq, int32_t Hq, int32_t causal_block,
                                         void *out, int64_t ldo, void *workspace, size_t ws_bytes,
                                         echo_stream_t stream) {
    using namespace echo;
    bool empty;
    const echo_status s = kv_check(pool, batch, &empty);
    if (s != ECHO_OK) return s;
    if (Hq < pool->H || Hq % pool->H || Hq / pool->H > 128 || causal_block < 0) return ECHO_ERR_SHAPE;
    if (ldq < (int64_t)Hq * pool->d || ldo < (int64_t)Hq * pool->d || ldq % 8 || ldo % 8)
        return ECHO_ERR_SHAPE;
    if (empty) return ECHO_OK;
    if (!q || !out || !workspace || !aligned16(q) || !aligned16(out)) return ECHO_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return ECHO_ERR_INVALID_ARG;
    if (ws_bytes < echo_kv_attention_workspace_size(pool, batch, Hq)) return ECHO_ERR_WORKSPACE;
    if (!device_supported()) return ECHO_ERR_UNSUPPORTED;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const int64_t blocks = ((int64_t)batch->n_rows * Hq + kThreads / 32 - 1) / (kThreads / 32);
    const bool i8 = pool->kind == ECHO_CACHE_INT8;
    auto kernel = pool->d == 64 ? (i8 ? kv_attention_kernel<true, 64> : kv_attention_kernel<false, 64>)
                                : (i8 ? kv_attention_kernel<true, 128> : kv_attention_kernel<false, 128>);
    LaunchScope ls(ECHO_K_KV_ATTENTION, batch->n_rows, (int64_t)Hq * pool->d, 0, st);
    launch_chained(kernel, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(kThreads), 0, st,
                   kv_pool(*pool), kv_batch(*batch), static_cast<const __nv_bfloat16 *>(q), ldq, Hq,
                   causal_block, 1.4426950408889634f / sqrtf((float)pool->d),
                   static_cast<__nv_bfloat16 *>(out), ldo, device_error_ptr());
    return last_launch_status();
}
