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
constexpr float kSeventh = (float)((1.0 - 1.0 / 1048576) / 7.0);   // 1 / 7, less 2^-20 of it

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

// place of row r in the pool, as kv_place: by the slot map where there is one; -1: none
ECHO_DEV int64_t row_place(const KvPool &pool, const KvBatch &b, const int64_t *place, int r, int *err) {
    if (place) {
        const int64_t at = place[r];
        if (at >> pool.shift < pool.n_pages) return at;      // -1 .. : left out
        echo_flag_error(err, ECHO_ERR_PAGE);
        return -1;
    }
    const KvRow row = kv_find_row(b, r);
    return row.seq < 0 || row.p < 0 ? -1 : kv_place(pool, b, row.seq, row.p, err);
}

// rows' keys and values into the pages: piece c of a row is EP values of its keys first and
// then of its values.  int8: 16, so that a division and the head's maximum (by shuffles) are
// few beside the values; with 8, rintf and casts, 32760 rows of 40 heads of 128 took 272 us,
// now 182.  A lane's values are 16-byte groups apart by the head's lanes, so that a warp
// reads and writes whole stretches.
template <typename T, int FORM, int D>
__global__ void __launch_bounds__(kThreads)
kv_write_kernel(const KvPool pool, const KvBatch b, const int64_t *__restrict__ place, const T *__restrict__ k,
                const T *__restrict__ v, int64_t ld, int *err) {
    pdl_enter();
    constexpr bool INT8 = FORM == kInt8;
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
        const int64_t at = row_place(pool, b, place, r, err);
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
                    static_cast<float *>(pool.scale)[vec] = !bad ? __fdiv_rn(amax, 127.f)
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

// The same into 4-bit pages: 8 neighbouring columns of a lane, four lanes to a scale.  Values are
// taken in bf16 first, so that max |u| / 7 and u / s have few bits and no division is needed: a product
// with 1 / 7 a little too small (2^-20) lies below a number of 5 bits where the quotient is that number, and
// above no other that the quotient is below; with 1 / s a little too large, the halves between two codes,
// and nothing else, pass over to the larger one.  (bf16 has 8 bits: other quotients are 2^-9 of
// themselves away.)  With divisions, and codes put together one by one, 32760 rows of 40 heads of 128 took
// 205 us, with an address made of the page for every store 160, now 140 (134 by a slot map; 127 at the rate of a
// copy).
ECHO_DEV uint32_t max_abs2(uint32_t a, uint32_t b) {      // of pairs, but for the signs; NaN where there is one
    uint32_t r;
    asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
ECHO_DEV float rcp_approx(float x) {                      // to 2^-23
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
kv_write4_kernel(const KvPool pool, const KvBatch b, const int64_t *__restrict__ place, const T *__restrict__ k,
                 const T *__restrict__ v, int64_t ld, int *err) {
    pdl_enter();
    constexpr int NG = 8 / kPer16<T>, U = kLoads / NG;
    constexpr uint32_t LPH = D / 8;
    const uint32_t lane = threadIdx.x & 31;
    const uint32_t half = pool.H * LPH, C = 2 * half;      // pieces of a row
    const uint32_t tasks = (C + 32 * U - 1) / (32 * U);
    const uint32_t code_step = (uint32_t)(D / 2) << pool.shift, scale_step = (uint32_t)(D / 32) << pool.shift;   // of a head
    PieceWalk walk(blockIdx.x * kWarps + (threadIdx.x >> 5), gridDim.x * kWarps, tasks);
    for (; walk.below(b.n_rows); walk.next()) {
        const int r = (int)walk.row;
        const uint32_t c0 = (uint32_t)walk.piece * 32 * U + lane;
        const T *const kr = k + r * ld, *const vr = v + r * ld - (int64_t)half * 8;    // piece c: 8 c from either
        uint4 in[U][NG];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t c = c0 + 32 * u;
#pragma unroll
            for (int h = 0; h < NG; ++h) {
                in[u][h] = make_uint4(0u, 0u, 0u, 0u);
                if (c < C) in[u][h] = __ldcs(reinterpret_cast<const uint4 *>((c < half ? kr : vr) + (uint64_t)c * 8) + h);
            }
        }
        const int64_t at = row_place(pool, b, place, r, err);
        if (at < 0) continue;
        // this token of the page's first head; heads, the values' after the keys', lie a step apart
        const int64_t vec = ((at >> pool.shift) * 2 * pool.H << pool.shift) + (at & ((1 << pool.shift) - 1));
        uint8_t *const codes_at = pool.pages + vec * (D / 2);
        uint16_t *const scales_at = static_cast<uint16_t *>(pool.scale) + vec * (D / 32);
        bool any = false;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t c = c0 + 32 * u;
            uint4 w = in[u][0];                       // 8 values in bf16
            if constexpr (NG == 2) {
                float f[8];
                values16<T>(in[u][0], f);
                values16<T>(in[u][NG - 1], f + 4);
                w = pack8_bf16(f);
            }
            const uint32_t pair[4] = {w.x, w.y, w.z, w.w};
            uint32_t a2 = max_abs2(max_abs2(w.x, w.y), max_abs2(w.z, w.w));
            a2 = max_abs2(a2, __shfl_xor_sync(0xffffffffu, a2, 1));
            a2 = max_abs2(a2, __shfl_xor_sync(0xffffffffu, a2, 2)) & 0x7FFF7FFFu;
            if (c >= C) continue;
            const uint32_t a = max(a2 << 16, a2 & 0xFFFF0000u);       // fp32 bits; NaN above infinity
            const bool bad = a >= 0x7F800000u;
            const float s = fmaxf(__uint_as_float((__float_as_uint(__fmul_rn(__uint_as_float(a), kSeventh)) + 0x7FFFFu) & ~0x7FFFFu),
                                  1.92592994438723585e-34f);          // 2^-112
            const float inv = __fmul_rn(rcp_approx(s), 1.f + 0x1p-20f);
            // 1.5 2^23 + 8 + code has the code, plus 8, in its low bits and nothing else below bit 22
            uint32_t even = 0, odd = 0;
#pragma unroll
            for (int i = 3; i >= 0; --i) {
                even = even * 16u + __float_as_uint(__fmaf_rn(bf16lo(pair[i]), inv, 12582920.f));
                odd = odd * 16u + __float_as_uint(__fmaf_rn(bf16hi(pair[i]), inv, 12582920.f));
            }
            const uint32_t codes = bad ? 0x88888888u : __byte_perm(even, odd, 0x5410);
            const uint32_t head = c / LPH, piece = c % LPH;
            *reinterpret_cast<uint32_t *>(codes_at + (uint64_t)head * code_step + piece * 4) = codes;
            // the scale's low 16 bits are zeros; what is not finite stands as it is
            if ((lane & 3) == 0)
                scales_at[(uint64_t)head * scale_step + piece / 4] = (uint16_t)((bad ? a : __float_as_uint(s)) >> 16);
            any |= bad;
        }
        if (any) echo_flag_error(err, ECHO_ERR_NONFINITE);
    }
}

// cached rows back: piece c of a row is 16 bytes of what is stored, so that a warp stores
// whole stretches
template <typename T, int FORM, int D>
__global__ void __launch_bounds__(kThreads)
kv_read_kernel(const KvPool pool, const KvBatch b, T *__restrict__ k, T *__restrict__ v, int64_t ld,
               int *err) {
    pdl_enter();
    constexpr bool INT8 = FORM == kInt8, INT4 = FORM == kInt4;
    constexpr int EP = kPer16<T>, BYTES = kv_bytes(FORM, EP), U = BYTES == 16 ? kLoads : 2 * kLoads;
    constexpr int WORDS = (BYTES + 3) / 4;
    constexpr uint32_t LPH = D / EP;
    const uint32_t lane = threadIdx.x & 31;
    const uint32_t half = pool.H * LPH, C = 2 * half;
    const uint32_t head_step = (uint32_t)kv_bytes(FORM, D) << pool.shift;
    const uint32_t tasks = (C + 32 * U - 1) / (32 * U);
    PieceWalk walk(blockIdx.x * kWarps + (threadIdx.x >> 5), gridDim.x * kWarps, tasks);
    for (; walk.below(b.n_rows); walk.next()) {
        const int r = (int)walk.row;
        const uint32_t c0 = (uint32_t)walk.piece * 32 * U + lane;
        const KvRow row = kv_find_row(b, r);
        if (row.seq < 0) continue;
        const int64_t at = row.p < 0 ? -1 : kv_place(pool, b, row.seq, row.p, err);   // -1: zeros
        // this token of the page's first head; heads, the values' after the keys', lie a step apart
        const int64_t vec0 = ((at >> pool.shift) * 2 * pool.H << pool.shift) + (at & ((1 << pool.shift) - 1));
        const uint8_t *const from = pool.pages + vec0 * kv_bytes(FORM, D);
        T *const kr = k + r * ld, *const vr = v + r * ld - (int64_t)half * EP;    // piece c: EP c from either
        uint32_t in[U][WORDS];
        float sc[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t c = c0 + 32 * u;
#pragma unroll
            for (int i = 0; i < WORDS; ++i) in[u][i] = INT4 ? 0x88888888u : 0u;      // codes 0
            sc[u] = 0.f;
            if (c >= C || at < 0) continue;
            const uint32_t head = c / LPH, piece = c % LPH;
            const uint8_t *src = from + (uint64_t)head * head_step + (INT4 ? piece * EP / 8 * 4 : piece * BYTES);
            if constexpr (BYTES == 16) {
                const uint4 w = __ldcs(reinterpret_cast<const uint4 *>(src));
                in[u][0] = w.x, in[u][1] = w.y, in[u][2] = w.z, in[u][3] = w.w;
            } else if constexpr (BYTES == 8) {
                const uint2 w = __ldcs(reinterpret_cast<const uint2 *>(src));
                in[u][0] = w.x, in[u][1] = w.y;
            } else {
                in[u][0] = __ldcs(reinterpret_cast<const uint32_t *>(src));
            }
            if constexpr (INT8) sc[u] = (static_cast<const float *>(pool.scale) + vec0)[(uint64_t)head << pool.shift];
            if constexpr (INT4)
                sc[u] = __uint_as_float((uint32_t)(static_cast<const uint16_t *>(pool.scale) + vec0 * (D / 32))
                                            [(uint64_t)head * ((D / 32u) << pool.shift) + piece * EP / 32] << 16);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t c = c0 + 32 * u;
            if (c >= C) continue;
            T *dst = (c >= half ? vr : kr) + (uint64_t)c * EP;
            float f[EP];
            if constexpr (INT4) {
                // code / 64, times 64, times the scale: exact.  fp32: four of a word's columns a lane
                const uint32_t s2 = __float_as_uint(sc[u]) | __float_as_uint(sc[u]) >> 16;
                const uint32_t w0 = EP == 8 ? in[u][0] : in[u][0] >> (8 * (c & 1));
                auto value2 = [&](uint32_t code) { return bf16x2_mul(bf16x2_mul(code, 0x42804280u), s2); };
                const uint4 w = make_uint4(value2(kv_nibbles2<0>(w0)), value2(kv_nibbles2<1>(w0)),
                                           value2(kv_nibbles2<2>(w0)), value2(kv_nibbles2<3>(w0)));
                if constexpr (sizeof(T) == 2) {
                    __stcs(reinterpret_cast<uint4 *>(dst), w);
                } else {
                    f[0] = bf16lo(w.x);
                    f[1] = bf16hi(w.x);
                    f[2] = bf16lo(w.y);
                    f[3] = bf16hi(w.y);
                    store16<T>(dst, f);
                }
                continue;
            }
#pragma unroll
            for (int i = 0; i < EP; ++i) {
                if constexpr (INT8) f[i] = __fmul_rn((float)(int8_t)(in[u][i >> 2] >> (8 * (i & 3))), sc[u]);
                else f[i] = i & 1 ? bf16hi(in[u][i >> 1]) : bf16lo(in[u][i >> 1]);
            }
            store16<T>(dst, f);
        }
    }
}

// blocks for the warps' tasks of all rows: `unroll` pieces of `values` a lane; a few waves at most
int grid_for(const echo_kv_pool &p, int n_rows, int values, int unroll) {
    const int64_t C = 2ll * p.H * p.d / values;
    const int64_t blocks = ((C + 32 * unroll - 1) / (32 * unroll) * n_rows + kWarps - 1) / kWarps;
    return (int)(blocks < 16384 ? blocks : 16384);
}

template <typename T, int FORM>
void launch_write(const echo_kv_pool &p, const echo_kv_batch &b, const int64_t *place, const void *k,
                  const void *v, int64_t ld, cudaStream_t st) {
    constexpr int EP = FORM == kInt8 ? 16 : 8;
    const int grid = grid_for(p, b.n_rows, EP, kLoads * kPer16<T> / EP);
    auto go = [&](auto *kernel) {
        echo::launch_chained(kernel, dim3(grid), dim3(kThreads), 0, st, echo::kv_pool(p), echo::kv_batch(b), place,
                             static_cast<const T *>(k), static_cast<const T *>(v), ld, echo::device_error_ptr());
    };
    if constexpr (FORM == kInt4) go(p.d == 64 ? kv_write4_kernel<T, 64> : kv_write4_kernel<T, 128>);
    else go(p.d == 64 ? kv_write_kernel<T, FORM, 64> : kv_write_kernel<T, FORM, 128>);
}

template <typename T>
echo_status write_rows(const echo_kv_pool &p, const echo_kv_batch &b, const int64_t *place, const void *k,
                       const void *v, int64_t ld, cudaStream_t st) {
    echo::LaunchScope ls(ECHO_K_KV_WRITE, b.n_rows, (int64_t)p.H * p.d, 0, st);
    if (p.kind == kInt4) launch_write<T, kInt4>(p, b, place, k, v, ld, st);
    else if (p.kind == kInt8) launch_write<T, kInt8>(p, b, place, k, v, ld, st);
    else launch_write<T, kBf16>(p, b, place, k, v, ld, st);
    return echo::last_launch_status();
}

template <typename T, int FORM>
void launch_read(const echo_kv_pool &p, const echo_kv_batch &b, void *k, void *v, int64_t ld,
                 cudaStream_t st) {
    const int grid = grid_for(p, b.n_rows, kPer16<T>, FORM == kBf16 && sizeof(T) == 2 ? kLoads : 2 * kLoads);
    echo::launch_chained(p.d == 64 ? kv_read_kernel<T, FORM, 64> : kv_read_kernel<T, FORM, 128>,
                         dim3(grid), dim3(kThreads), 0, st, echo::kv_pool(p), echo::kv_batch(b),
                         static_cast<T *>(k), static_cast<T *>(v), ld, echo::device_error_ptr());
}

template <typename T>
echo_status read_rows(const echo_kv_pool &p, const echo_kv_batch &b, void *k, void *v, int64_t ld, cudaStream_t st) {
    echo::LaunchScope ls(ECHO_K_KV_READ, b.n_rows, (int64_t)p.H * p.d, 0, st);
    if (p.kind == kInt4) launch_read<T, kInt4>(p, b, k, v, ld, st);
    else if (p.kind == kInt8) launch_read<T, kInt8>(p, b, k, v, ld, st);
    else launch_read<T, kBf16>(p, b, k, v, ld, st);
    return echo::last_launch_status();
}

echo_status check_tensors(const echo_kv_pool *pool, const void *k, const void *v, int64_t ld, echo_dtype t,
                          bool empty) {
    if (t != ECHO_BF16 && t != ECHO_F32) return ECHO_ERR_INVALID_ARG;
    if (ld < (int64_t)pool->H * pool->d || ld % 8) return ECHO_ERR_SHAPE;
    if (empty) return ECHO_OK;
    if (!k || !v || !echo::aligned16(k) || !echo::aligned16(v)) return ECHO_ERR_INVALID_ARG;
    return echo::device_supported() ? ECHO_OK : ECHO_ERR_UNSUPPORTED;
}

echo_status check_rows(const echo_kv_pool *pool, const echo_kv_batch *batch, const void *k,
                       const void *v, int64_t ld, echo_dtype t, bool *empty) {
    echo_status s = echo::kv_check(pool, batch, empty);
    if (s != ECHO_OK) return s;
    return check_tensors(pool, k, v, ld, t, *empty);
}

}  // namespace

namespace echo {

static echo_status pool_sizes(const echo_kv_pool *p) {
    if (p->kind != kInt8 && p->kind != kBf16 && p->kind != kInt4) return ECHO_ERR_INVALID_ARG;
    if (p->n_pages < 1 || p->H < 1 || (p->d != 64 && p->d != 128)) return ECHO_ERR_SHAPE;
    if (p->page_tokens != 16 && p->page_tokens != 32 && p->page_tokens != 64 && p->page_tokens != 128)
        return ECHO_ERR_SHAPE;
    // a (page, keys or values, head) is one 32-bit coordinate of the tensor maps
    return 2ll * p->n_pages * p->H > INT32_MAX - 1 ? ECHO_ERR_SHAPE : ECHO_OK;
}

static echo_status pool_memory(const echo_kv_pool *p) {
    if (!p->pages || !aligned16(p->pages)) return ECHO_ERR_INVALID_ARG;
    if (p->kind != kBf16 && (!p->scale || !aligned16(p->scale))) return ECHO_ERR_INVALID_ARG;
    return ECHO_OK;
}

echo_status kv_check(const echo_kv_pool *p, const echo_kv_batch *b, bool *empty) {
    if (!p || !b) return ECHO_ERR_INVALID_ARG;
    echo_status s = pool_sizes(p);
    if (s != ECHO_OK) return s;
    if (b->n_seqs < 0 || b->max_pages < 0 || b->n_rows < 0 || b->max_rows < 0 || b->max_len < 0) return ECHO_ERR_SHAPE;
    if ((s = pool_memory(p)) != ECHO_OK) return s;
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
    return t == ECHO_BF16 ? write_rows<__nv_bfloat16>(*pool, *batch, nullptr, k, v, ld, st)
                          : write_rows<float>(*pool, *batch, nullptr, k, v, ld, st);
}

extern "C" echo_status echo_kv_write_at(const echo_kv_pool *pool, const int64_t *place, int32_t n_rows,
                                        const void *k, const void *v, int64_t ld, echo_dtype t,
                                        echo_stream_t stream) {
    if (!pool) return ECHO_ERR_INVALID_ARG;
    echo_status s = echo::pool_sizes(pool);
    if (s != ECHO_OK) return s;
    if (n_rows < 0) return ECHO_ERR_SHAPE;
    if ((s = echo::pool_memory(pool)) != ECHO_OK) return s;
    if (n_rows > 0 && (!place || (reinterpret_cast<uintptr_t>(place) & 7u))) return ECHO_ERR_INVALID_ARG;
    s = check_tensors(pool, k, v, ld, t, n_rows == 0);
    if (s != ECHO_OK || n_rows == 0) return s;
    echo_kv_batch b = {};
    b.n_rows = n_rows;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    return t == ECHO_BF16 ? write_rows<__nv_bfloat16>(*pool, b, place, k, v, ld, st)
                          : write_rows<float>(*pool, b, place, k, v, ld, st);
}

extern "C" echo_status echo_kv_read(const echo_kv_pool *pool, const echo_kv_batch *batch, void *k,
                                    void *v, int64_t ld, echo_dtype t, echo_stream_t stream) {
    bool empty;
    const echo_status s = check_rows(pool, batch, k, v, ld, t, &empty);
    if (s != ECHO_OK || empty) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    return t == ECHO_BF16 ? read_rows<__nv_bfloat16>(*pool, *batch, k, v, ld, st)
                          : read_rows<float>(*pool, *batch, k, v, ld, st);
}
