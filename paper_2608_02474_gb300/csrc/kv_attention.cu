// Attention of new rows over the paged key/value cache: the entry point.
#include "kv_pages.cuh"

namespace {
echo_status check_sizes(const echo_kv_pool *pool, const echo_kv_batch *batch, int32_t Hq, bool *empty) {
    const echo_status s = echo::kv_check(pool, batch, empty);
    if (s != ECHO_OK) return s;
    if (Hq < pool->H || Hq % pool->H || Hq / pool->H > 128) return ECHO_ERR_SHAPE;
    return (int64_t)batch->n_rows * Hq > INT32_MAX ? ECHO_ERR_SHAPE : ECHO_OK;
}
}  // namespace

extern "C" size_t echo_kv_attention_workspace_size(const echo_kv_pool *pool, const echo_kv_batch *batch,
                                                   int32_t Hq) {
    bool empty;
    if (check_sizes(pool, batch, Hq, &empty) != ECHO_OK) return 0;
    const size_t few = echo::kv_decode_workspace(*pool), many = echo::kv_chunk_workspace(*pool);
    return few > many ? few : many;
}

extern "C" echo_status echo_kv_attention(const echo_kv_pool *pool, const echo_kv_batch *batch,
                                         const void *q, int64_t ldq, int32_t Hq, int32_t causal_block,
                                         void *out, int64_t ldo, void *workspace, size_t ws_bytes,
                                         echo_stream_t stream) {
    using namespace echo;
    bool empty;
    const echo_status s = check_sizes(pool, batch, Hq, &empty);
    if (s != ECHO_OK) return s;
    if (causal_block < 0) return ECHO_ERR_SHAPE;
    if (ldq < (int64_t)Hq * pool->d || ldo < (int64_t)Hq * pool->d || ldq % 8 || ldo % 8)
        return ECHO_ERR_SHAPE;
    if (empty) return ECHO_OK;
    if (!q || !out || !workspace || !aligned16(q) || !aligned16(out)) return ECHO_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return ECHO_ERR_INVALID_ARG;
    if (ws_bytes < echo_kv_attention_workspace_size(pool, batch, Hq)) return ECHO_ERR_WORKSPACE;
    if (!device_supported()) return ECHO_ERR_UNSUPPORTED;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const KvAttention a{pool, batch, q, ldq, Hq, causal_block, out, ldo, workspace};
    const int64_t rows = (int64_t)batch->max_rows * (Hq / pool->H);   // packed, of a sequence
    return kv_few_rows(*pool, rows) ? launch_kv_decode(a, rows, st) : launch_kv_chunk(a, st);
}
