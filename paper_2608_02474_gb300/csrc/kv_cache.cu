// The paged key/value cache: new rows written into pages (rounded to bf16, or
// quantised to int8 with a scale per token and head) and cached rows read back.
//
// Both are one pass: a value is read once and written once, and the time is that of
// the bytes.  A warp takes some of one row's pieces, so that its loads are all in flight
// before the first is used, and finds the row's place in the pool meanwhile.  A head's
// values lie in neighbouring lanes, which gives its maximum by their shuffles.
#include "kv_pages.cuh"

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kLoads = 4;   // 16-byte loads of a lane on their way at once

// 16 bytes of a row: 8 bf16 values, or 4 of fp32
template <typename T>
constexpr int kPer16 = 16 / (int)sizeof(T);
template <typename T>
ECHO_DEV void values16(const uint4 &v, float *f) {
    if constexpr (sizeof(T) == 2) {
        unpack8_bf16(v, f);
    } else {
        f[0] = __uint_as_float(v.x);
        f[1] = __uint_as_float(v.y);
        f[2] = __uint_as_float(v.z);
        f[3] = __uint_as_float(v.w);
    }
}
template <typename T>
ECHO_DEV void store16(T *p, const float *f) {
    if constexpr (sizeof(T) == 2) __stcs(reinterpret_cast<uint4 *>(p), pack8_bf16(f));
    else __stcs(reinterpret_cast<float4 *>(p), make_float4(f[0], f[1], f[2], f[3]));
}

// Codes without conversions, which run at an eighth of the rate of additions:
// 1.5 2^23 + t, |t| < 2^22, is 1.5 2^23 + rint(t) (half to even), with rint(t) in two's
// complement in its low bits; |v inv| stays below 127.5 for a finite inv, so that nothing is
// clamped.
ECHO_DEV uint32_t codes4(const float *f, float inv) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(__fadd_rn(__fmul_rn(f[i], inv), 12582912.f));
    return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
}

// rows' keys and values into the pages: piece c of a row is EP values of its keys first and
// then of its values.  int8: 16, so that a division and the head's maximum (by shuffles) are
// few beside the values; with 8, rintf and casts, 32760 rows of 40 heads of 128 took 272 us,
// now 182.  A lane's values are 16-byte groups apart by the head's lanes, so that a warp
// reads and writes whole stretches.
template <typename T, bool INT8, int D>
__global__ void __launch_bounds__(kThreads)
kv_write_kernel(const KvPool pool, const KvBatch b, const T *__restrict__ k, const T *__restrict__ v,
                int64_t ld, int *err) {
    pdl_enter();
    constexpr int GE = kPer16<T>, EP = INT8 ? 16 : 8, NG = EP / GE, LPH = D / EP;   // lanes of a head
    constexpr int U = kLoads / NG;
    const int lane = threadIdx.x & 31;
    const int half = pool.H * LPH, C = 2 * half;      // pieces of a row
    const int tasks = (C + 32 * U - 1) / (32 * U);
    PieceWalk walk(blockIdx.x * kWarps + (threadIdx.x >> 5), gridDim.x * kWarps, tasks);
    for (; walk.below(b.n_rows); walk.next()) {
        const int r = (int)walk.row, c0 = (int)walk.piece * 32 * U + lane;
        uint4 in[U][NG];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + 32 * u, ch = c < half ? c : c - half;
            if (c < C) {
                const T *src = (c < half ? k : v) + r * ld + (ch / LPH) * D + (ch % LPH) * GE;
#pragma unroll
                for (int h = 0; h < NG; ++h) in[u][h] = __ldcs(reinterpret_cast<const uint4 *>(src + h * (D / NG)));
            }
        }
        const KvRow row = kv_find_row(b, r);
        if (row.seq < 0 || row.p < 0) continue;
        const int64_t at = kv_place(pool, b, row.seq, row.p, err);
        if (at < 0) continue;
        const int64_t page = at >> pool.shift, slot = at & ((1 << pool.shift) - 1);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + 32 * u;
            const int kv = c >= half, ch = kv ? c - half : c;
            const int64_t vec = (((page * 2 + kv) * pool.H + ch / LPH) << pool.shift) + slot;
            float f[EP] = {};
            if (c < C) {
#pragma unroll
                for (int h = 0; h < NG; ++h) values16<T>(in[u][h], f + h * GE);
            }
            if constexpr (INT8) {
                // the largest |value| as fp32 bits: infinity above every number, NaN above it
                uint32_t a = 0;
#pragma unroll
                for (int i = 0; i < EP; ++i) a = max(a, __float_as_uint(f[i]) & 0x7FFFFFFFu);
#pragma unroll
                for (int o = LPH / 2; o > 0; o >>= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
                if (c >= C) continue;
                const bool bad = a >= 0x7F800000u;
                const float amax = __uint_as_float(a);
                float inv = !bad && amax > 0.f ? __fdiv_rn(127.f, amax) : 0.f;
                if (inv == INFINITY) {          // amax below 3.7e-37: +-127 by the clamp, and 0
                    inv = 127.f;
#pragma unroll
                    for (int i = 0; i < EP; ++i) f[i] = f[i] == 0.f ? 0.f : copysignf(1.f, f[i]);
                }
                uint8_t *dst = pool.pages + vec * D + (ch % LPH) * GE;
#pragma unroll
                for (int h = 0; h < NG; ++h) {
                    const uint32_t lo = bad ? 0u : codes4(f + h * GE, inv);
                    if constexpr (GE == 4) {
                        *reinterpret_cast<uint32_t *>(dst + h * (D / NG)) = lo;
                    } else {
                        *reinterpret_cast<uint2 *>(dst + h * (D / NG)) =
                            make_uint2(lo, bad ? 0u : codes4(f + h * GE + 4, inv));
                    }
                }
                if (ch % LPH == 0) {
                    pool.scale[vec] = !bad ? __fdiv_rn(amax, 127.f)
                                           : a > 0x7F800000u ? __int_as_float(0x7fc00000) : INFINITY;
                    if (bad) echo_flag_error(err, ECHO_ERR_NONFINITE);
                }
            } else if (c < C) {
                uint8_t *dst = pool.pages + (vec * D + (ch % LPH) * GE) * 2;
#pragma unroll
                for (int h = 0; h < NG; ++h) {
                    if constexpr (GE == 8) {
                        *reinterpret_cast<uint4 *>(dst) = in[u][0];
                    } else {
                        *reinterpret_cast<uint2 *>(dst + h * D) =
                            make_uint2(pack_bf16(f[4 * h], f[4 * h + 1]), pack_bf16(f[4 * h + 2], f[4 * h + 3]));
                    }
                }
            }
        }
    }
}

// cached rows back: piece c of a row is 16 bytes of what is stored, so that a warp stores
// whole stretches
template <typename T, bool INT8, int D>
__global__ void __launch_bounds__(kThreads)
kv_read_kernel(const KvPool pool, const KvBatch b, T *__restrict__ k, T *__restrict__ v, int64_t ld,
               int *err) {
    pdl_enter();
    constexpr int EP = kPer16<T>, BYTES = EP * (INT8 ? 1 : 2), LPH = D / EP, U = BYTES == 16 ? kLoads : 2 * kLoads;
    const int lane = threadIdx.x & 31;
    const int half = pool.H * LPH, C = 2 * half;
    const int tasks = (C + 32 * U - 1) / (32 * U);
    PieceWalk walk(blockIdx.x * kWarps + (threadIdx.x >> 5), gridDim.x * kWarps, tasks);
    for (; walk.below(b.n_rows); walk.next()) {
        const int r = (int)walk.row, c0 = (int)walk.piece * 32 * U + lane;
        const KvRow row = kv_find_row(b, r);
        if (row.seq < 0) continue;
        const int64_t at = row.p < 0 ? -1 : kv_place(pool, b, row.seq, row.p, err);   // -1: zeros
        const int64_t page = at >> pool.shift, slot = at & ((1 << pool.shift) - 1);
        uint32_t in[U][BYTES / 4];
        float sc[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + 32 * u;
#pragma unroll
            for (int i = 0; i < BYTES / 4; ++i) in[u][i] = 0u;
            sc[u] = 0.f;
            if (c >= C || at < 0) continue;
            const int kv = c >= half, ch = kv ? c - half : c;
            const int64_t vec = (((page * 2 + kv) * pool.H + ch / LPH) << pool.shift) + slot;
            const uint8_t *src = pool.pages + vec * D * (INT8 ? 1 : 2) + ch % LPH * BYTES;
            if constexpr (BYTES == 16) {
                const uint4 w = __ldcs(reinterpret_cast<const uint4 *>(src));
                in[u][0] = w.x, in[u][1] = w.y, in[u][2] = w.z, in[u][3] = w.w;
            } else if constexpr (BYTES == 8) {
                const uint2 w = __ldcs(reinterpret_cast<const uint2 *>(src));
                in[u][0] = w.x, in[u][1] = w.y;
            } else {
                in[u][0] = __ldcs(reinterpret_cast<const uint32_t *>(src));
            }
            if constexpr (INT8) sc[u] = pool.scale[vec];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + 32 * u;
            if (c >= C) continue;
            float f[EP];
#pragma unroll
            for (int i = 0; i < EP; ++i) {
                if constexpr (INT8) f[i] = __fmul_rn((float)(int8_t)(in[u][i >> 2] >> (8 * (i & 3))), sc[u]);
                else f[i] = i & 1 ? bf16hi(in[u][i >> 1]) : bf16lo(in[u][i >> 1]);
            }
            store16<T>((c >= half ? v : k) + r * ld + (int64_t)(c >= half ? c - half : c) * EP, f);
        }
    }
}

// blocks for the warps' tasks of all rows: `unroll` pieces of `values` a lane; a few waves at most
int grid_for(const echo_kv_pool &p, int n_rows, int values, int unroll) {
    const int64_t C = 2ll * p.H * p.d / values;
    const int64_t blocks = ((C + 32 * unroll - 1) / (32 * unroll) * n_rows + kWarps - 1) / kWarps;
    return (int)(blocks < 16384 ? blocks : 16384);
}

template <typename T, bool INT8>
void launch_write(const echo_kv_pool &p, const echo_kv_batch &b, const void *k, const void *v,
                  int64_t ld, cudaStream_t st) {
    constexpr int EP = INT8 ? 16 : 8;
    const int grid = grid_for(p, b.n_rows, EP, kLoads * kPer16<T> / EP);
    echo::launch_chained(p.d == 64 ? kv_write_kernel<T, INT8, 64> : kv_write_kernel<T, INT8, 128>,
                         dim3(grid), dim3(kThreads), 0, st, echo::kv_pool(p), echo::kv_batch(b),
                         static_cast<const T *>(k), static_cast<const T *>(v), ld,
                         echo::device_error_ptr());
}

template <typename T, bool INT8>
void launch_read(const echo_kv_pool &p, const echo_kv_batch &b, void *k, void *v, int64_t ld,
                 cudaStream_t st) {
    const int grid = grid_for(p, b.n_rows, kPer16<T>, !INT8 && sizeof(T) == 2 ? kLoads : 2 * kLoads);
    echo::launch_chained(p.d == 64 ? kv_read_kernel<T, INT8, 64> : kv_read_kernel<T, INT8, 128>,
                         dim3(grid), dim3(kThreads), 0, st, echo::kv_pool(p), echo::kv_batch(b),
                         static_cast<T *>(k), static_cast<T *>(v), ld, echo::device_error_ptr());
}

echo_status check_rows(const echo_kv_pool *pool, const echo_kv_batch *batch, const void *k,
                       const void *v, int64_t ld, echo_dtype t, bool *empty) {
    const echo_status s = echo::kv_check(pool, batch, empty);
    if (s != ECHO_OK) return s;
    if (t != ECHO_BF16 && t != ECHO_F32) return ECHO_ERR_INVALID_ARG;
    if (ld < (int64_t)pool->H * pool->d || ld % 8) return ECHO_ERR_SHAPE;
    if (*empty) return ECHO_OK;
    if (!k || !v || !echo::aligned16(k) || !echo::aligned16(v)) return ECHO_ERR_INVALID_ARG;
    return echo::device_supported() ? ECHO_OK : ECHO_ERR_UNSUPPORTED;
}

}  // namespace

namespace echo {

echo_status kv_check(const echo_kv_pool *p, const echo_kv_batch *b, bool *empty) {
    if (!p || !b) return ECHO_ERR_INVALID_ARG;
    if (p->kind != ECHO_CACHE_INT8 && p->kind != ECHO_CACHE_BF16) return ECHO_ERR_INVALID_ARG;
    if (p->n_pages < 1 || p->H < 1 || (p->d != 64 && p->d != 128)) return ECHO_ERR_SHAPE;
    if (p->page_tokens != 16 && p->page_tokens != 32 && p->page_tokens != 64 && p->page_tokens != 128)
        return ECHO_ERR_SHAPE;
    // a (page, keys or values, head) is one 32-bit coordinate of the tensor maps
    if (2ll * p->n_pages * p->H > INT32_MAX - 1) return ECHO_ERR_SHAPE;
    if (b->n_seqs < 0 || b->max_pages < 0 || b->n_rows < 0 || b->max_rows < 0) return ECHO_ERR_SHAPE;
    if (!p->pages || !aligned16(p->pages)) return ECHO_ERR_INVALID_ARG;
    if (p->kind == ECHO_CACHE_INT8 && (!p->scale || !aligned16(p->scale))) return ECHO_ERR_INVALID_ARG;
    *empty = b->n_seqs == 0 || b->n_rows == 0;
    if (*empty) return ECHO_OK;
    auto aligned4 = [](const void *q) { return (reinterpret_cast<uintptr_t>(q) & 3u) == 0; };
    if (!b->len || !b->row0 || !aligned4(b->len) || !aligned4(b->row0)) return ECHO_ERR_INVALID_ARG;
    if (b->max_pages > 0 && (!b->table || !aligned4(b->table))) return ECHO_ERR_INVALID_ARG;
    return ECHO_OK;
}

}  // namespace echo

extern "C" echo_status echo_kv_write(const echo_kv_pool *pool, const echo_kv_batch *batch,
                                     const void *k, const void *v, int64_t ld, echo_dtype t,
                                     echo_stream_t stream) {
    bool empty;
    const echo_status s = check_rows(pool, batch, k, v, ld, t, &empty);
    if (s != ECHO_OK || empty) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    echo::LaunchScope ls(ECHO_K_KV_WRITE, batch->n_rows, (int64_t)pool->H * pool->d, 0, st);
    const bool q = pool->kind == ECHO_CACHE_INT8;
    if (t == ECHO_BF16)
        q ? launch_write<__nv_bfloat16, true>(*pool, *batch, k, v, ld, st)
          : launch_write<__nv_bfloat16, false>(*pool, *batch, k, v, ld, st);
    else
        q ? launch_write<float, true>(*pool, *batch, k, v, ld, st)
          : launch_write<float, false>(*pool, *batch, k, v, ld, st);
    return echo::last_launch_status();
}

extern "C" echo_status echo_kv_read(const echo_kv_pool *pool, const echo_kv_batch *batch, void *k,
                                    void *v, int64_t ld, echo_dtype t, echo_stream_t stream) {
    bool empty;
    const echo_status s = check_rows(pool, batch, k, v, ld, t, &empty);
    if (s != ECHO_OK || empty) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    echo::LaunchScope ls(ECHO_K_KV_READ, batch->n_rows, (int64_t)pool->H * pool->d, 0, st);
    const bool q = pool->kind == ECHO_CACHE_INT8;
    if (t == ECHO_BF16)
        q ? launch_read<__nv_bfloat16, true>(*pool, *batch, k, v, ld, st)
          : launch_read<__nv_bfloat16, false>(*pool, *batch, k, v, ld, st);
    else
        q ? launch_read<float, true>(*pool, *batch, k, v, ld, st)
          : launch_read<float, false>(*pool, *batch, k, v, ld, st);
    return echo::last_launch_status();
}
