// The end of one branch of a block and the beginning of the next, row by row: the branch's
// output normed, gated and added to the residual stream, the result normed and modulated,
//   h = alpha x + beta gate * N_after(y),   n = N_before(h) * (1 + scale) + shift.
// One pass: a row's x and y are read once, h and n written once, and the time of many rows is
// that of those bytes (32760 bf16 rows of 5120: 1.34 GB in 211 us, 0.94 of a copy's rate), of few rows
// that of one access after the other.  Sums are fp32 trees over the row's threads, a mean first and then
// the centred squares.  gate, scale and shift (for fp32 as many bytes as a row's x, y, h and n, and half
// as many again) are read again only where the modulation changes.
#include <type_traits>

#include "common.cuh"
#include "internal.h"

namespace {

struct Norm {
    int kind;
    float eps;
    const float *weight, *bias;
};
struct NormParams {
    const void *x, *y;
    void *h, *n;
    const void *gate, *scale, *shift;
    const int32_t *mod_rows;
    int64_t ldx, ldy, ldh, ldn, ldm;
    Norm after, before;
    float alpha, beta, inv_d;
    int n_rows, chunks;                  // of 8 values
    int n_mods, rows_per_mod;            // n_mods < 0: no modulations
    bool xf, yf, hf, nf, mf;             // fp32, not bf16
};

// a row that is read once: past the L1
ECHO_DEV uint4 ld_once(const void *p) {
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}
ECHO_DEV void floats4(const uint4 &v, float *f) {
    f[0] = __uint_as_float(v.x);
    f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z);
    f[3] = __uint_as_float(v.w);
}

// the thread's chunks of a row; zeros past its end
template <int TPR, int CH>
ECHO_DEV void load_row(const void *p, int64_t at, bool f32, int t, int chunks, float (*v)[8]) {
    if (f32) {
        const float *src = static_cast<const float *>(p) + at;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = t + k * TPR;
            uint4 a = make_uint4(0, 0, 0, 0), b = a;
            if (c < chunks) {
                a = ld_once(src + 8 * c);
                b = ld_once(src + 8 * c + 4);
            }
            floats4(a, v[k]);
            floats4(b, v[k] + 4);
        }
    } else {
        const __nv_bfloat16 *src = static_cast<const __nv_bfloat16 *>(p) + at;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = t + k * TPR;
            uint4 a = make_uint4(0, 0, 0, 0);
            if (c < chunks) a = ld_once(src + 8 * c);
            unpack8_bf16(a, v[k]);
        }
    }
}
ECHO_DEV void store8(void *p, int64_t at, bool f32, const float *v) {
    if (f32) {
        float4 *dst = reinterpret_cast<float4 *>(static_cast<float *>(p) + at);
        dst[0] = make_float4(v[0], v[1], v[2], v[3]);
        dst[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
        *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p) + at) = pack8_bf16(v);
    }
}
// 8 values that rows share
ECHO_DEV void shared8(const void *p, int64_t at, bool f32, float *v) {
    if (f32) {
        const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const float *>(p) + at);
        floats4(__ldg(src), v);
        floats4(__ldg(src + 1), v + 4);
    } else {
        unpack8_bf16(__ldg(reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(p) + at)), v);
    }
}

// Sum over the row's threads.  Two buffers in turn: whoever writes one has passed the barrier
// of the sum between, and so have all readers of the sum before.
template <int TPR>
ECHO_DEV float row_sum(float v, float (*red)[TPR / 32], int &turn) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    float *at = red[turn & 1];
    ++turn;
    if ((threadIdx.x & 31) == 0) at[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 32; ++w) v += at[w];
    return v;
}

// mean (LAYER) and 1 / root of the row's spread; v is centred in place
template <int TPR, int CH>
ECHO_DEV float spread(const Norm &n, float inv_d, int t, int chunks, float (*v)[8], float (*red)[TPR / 32], int &turn) {
    if (n.kind == ECHO_NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < CH; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += v[k][e];
        const float mean = row_sum<TPR>(s, red, turn) * inv_d;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const bool live = t + k * TPR < chunks;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] = live ? v[k][e] - mean : 0.f;
        }
    }
    float ss = 0.f;
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += v[k][e] * v[k][e];
    return rsqrtf(row_sum<TPR>(ss, red, turn) * inv_d + n.eps);
}
ECHO_DEV void affine(const Norm &n, int c, float *v) {
    float w[8];
    if (n.weight) {
        shared8(n.weight, 8 * c, true, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= w[e];
    }
    if (n.bias) {
        shared8(n.bias, 8 * c, true, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += w[e];
    }
}

// Rows of more than 8192 values: a block to a row, CH chunks of 8 values a thread.
template <int TPR, int CH>
__global__ void __launch_bounds__(TPR)
gated_norm_kernel(const NormParams p) {
    pdl_enter();
    __shared__ float red[2][TPR / 32];
    const int t = threadIdx.x;
    const int first = (int)((int64_t)p.n_rows * blockIdx.x / gridDim.x);
    const int last = (int)((int64_t)p.n_rows * (blockIdx.x + 1) / gridDim.x);
    int turn = 0;
    for (int r = first; r < last; ++r) {
        int m = 0;
        if (p.n_mods >= 0) {
            m = p.mod_rows ? p.mod_rows[r] : r / p.rows_per_mod;
            if ((unsigned)m >= (unsigned)p.n_mods) continue;
        }
        float h[CH][8];
        load_row<TPR, CH>(p.x, r * p.ldx, p.xf, t, p.chunks, h);
        if (p.y) {
            float y[CH][8];
            load_row<TPR, CH>(p.y, r * p.ldy, p.yf, t, p.chunks, y);
            float f = p.beta;
            if (p.after.kind != ECHO_NORM_NONE) f = spread<TPR, CH>(p.after, p.inv_d, t, p.chunks, y, red, turn);
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const int c = t + k * TPR;
                if (c >= p.chunks) continue;
                if (p.after.kind != ECHO_NORM_NONE) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[k][e] *= f;
                    affine(p.after, c, y[k]);
                }
                float g[8];
                if (p.gate) shared8(p.gate, m * p.ldm + 8 * c, p.mf, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float b = p.gate ? p.beta * g[e] : p.beta;
                    h[k][e] = fmaf(b, y[k][e], p.alpha * h[k][e]);
                }
            }
        } else {
#pragma unroll
            for (int k = 0; k < CH; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) h[k][e] *= p.alpha;
        }
        if (p.h) {
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                const int c = t + k * TPR;
                if (c < p.chunks) store8(p.h, r * p.ldh + 8 * c, p.hf, h[k]);
            }
        }
        if (!p.n) continue;
        float f = 1.f;
        if (p.before.kind != ECHO_NORM_NONE) f = spread<TPR, CH>(p.before, p.inv_d, t, p.chunks, h, red, turn);
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            const int c = t + k * TPR;
            if (c >= p.chunks) continue;
            if (p.before.kind != ECHO_NORM_NONE) {
#pragma unroll
                for (int e = 0; e < 8; ++e) h[k][e] *= f;
                affine(p.before, c, h[k]);
            }
            float g[8];
            if (p.scale) {
                shared8(p.scale, m * p.ldm + 8 * c, p.mf, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[k][e] = fmaf(h[k][e], g[e], h[k][e]);
            }
            if (p.shift) {
                shared8(p.shift, m * p.ldm + 8 * c, p.mf, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[k][e] += g[e];
            }
            store8(p.n, r * p.ldn + 8 * c, p.nf, h[k]);
        }
    }
}

// Many rows: a chunk of 8 columns to a thread, so that its gate, scale and
// shift stay in registers while the rows' modulation is the same (the norms' weights in them), and R rows at
// a time, whose sums share their barriers.  Rows come by bulk copies into two buffers of R rows; a buffer
// is filled again as soon as its rows are in registers, while the sums of these are under way.
// A block takes neighbouring rows (in turn with the others, 264 us for 211: the modulation comes again and again).
constexpr int kBufferBytes = 100 * 1024;

// R sums over the block, in all threads.  A lane passes on half of what it holds at a time, so
// that R = 4 sums take 6 exchanges and not 20.
template <int R>
ECHO_DEV void block_sums(float (&v)[R], float4 (*part)[32], int &turn) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    auto reduce = [&](float a, float b, float c, float d) -> float {   // of row lane / 8
        const bool high = lane & 16;
        const float x = high ? c : a, y = high ? d : b;
        float s0 = x + __shfl_xor_sync(0xffffffffu, high ? a : c, 16), s1 = y + __shfl_xor_sync(0xffffffffu, high ? b : d, 16);
        const bool odd = lane & 8;
        float s = (odd ? s1 : s0) + __shfl_xor_sync(0xffffffffu, odd ? s0 : s1, 8);
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        return s;
    };
    float4 *at = part[turn & 1];
    ++turn;
    if constexpr (R == 1) {
        float s = v[0];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0) at[warp].x = s;
        __syncthreads();
        s = lane < warps ? at[lane].x : 0.f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        v[0] = s;
        return;
    }
    const float s = reduce(v[0], v[1 % R], R > 2 ? v[2 % R] : 0.f, R > 2 ? v[3 % R] : 0.f);
    if ((lane & 7) == 0) reinterpret_cast<float *>(&at[warp])[lane >> 3] = s;
    __syncthreads();
    const float4 w = lane < warps ? at[lane] : make_float4(0.f, 0.f, 0.f, 0.f);
    const float all = reduce(w.x, w.y, w.z, w.w);
#pragma unroll
    for (int k = 0; k < R; ++k) v[k] = __shfl_sync(0xffffffffu, all, 8 * k);
}

// Values in pairs: one instruction for two of them.
struct Pairs {
    uint64_t v[4];
};
ECHO_DEV Pairs splat(float x) { return {{f2_pack(x, x), f2_pack(x, x), f2_pack(x, x), f2_pack(x, x)}}; }
ECHO_DEV Pairs pairs_of(const float *f) {
    return {{f2_pack(f[0], f[1]), f2_pack(f[2], f[3]), f2_pack(f[4], f[5]), f2_pack(f[6], f[7])}};
}
ECHO_DEV void floats_of(const Pairs &p, float *f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f2_unpack(p.v[i], f[2 * i], f[2 * i + 1]);
}
ECHO_DEV Pairs fma8(const Pairs &a, const Pairs &b, const Pairs &c) {
    return {{f2_fma(a.v[0], b.v[0], c.v[0]), f2_fma(a.v[1], b.v[1], c.v[1]), f2_fma(a.v[2], b.v[2], c.v[2]), f2_fma(a.v[3], b.v[3], c.v[3])}};
}
ECHO_DEV Pairs mul8(const Pairs &a, const Pairs &b) {
    return {{f2_mul(a.v[0], b.v[0]), f2_mul(a.v[1], b.v[1]), f2_mul(a.v[2], b.v[2]), f2_mul(a.v[3], b.v[3])}};
}
ECHO_DEV Pairs add8(const Pairs &a, const Pairs &b) {
    return {{f2_add(a.v[0], b.v[0]), f2_add(a.v[1], b.v[1]), f2_add(a.v[2], b.v[2]), f2_add(a.v[3], b.v[3])}};
}
ECHO_DEV float sum8(const Pairs &a) {
    float x, y;
    f2_unpack(f2_add(f2_add(a.v[0], a.v[1]), f2_add(a.v[2], a.v[3])), x, y);
    return x + y;
}
ECHO_DEV float square8(const Pairs &a) {
    float x, y;
    f2_unpack(f2_add(f2_fma(a.v[0], a.v[0], f2_mul(a.v[1], a.v[1])), f2_fma(a.v[2], a.v[2], f2_mul(a.v[3], a.v[3]))), x, y);
    return x + y;
}
ECHO_DEV Pairs shared_pairs(const void *p, int64_t at, bool f32) {
    float f[8];
    shared8(p, at, f32, f);
    return pairs_of(f);
}

// R rows' chunks from shared memory; zeros past the row's end and the last row
template <int R, int N>
ECHO_DEV void staged(const uint8_t *rows, uint32_t row_bytes, bool f32, int t, int n, Pairs (&v)[N]) {
    if (f32) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            float f[8] = {};
            if (k < n) {
                floats4(reinterpret_cast<const uint4 *>(rows + k * row_bytes)[2 * t], f);
                floats4(reinterpret_cast<const uint4 *>(rows + k * row_bytes)[2 * t + 1], f + 4);
            }
            v[k] = pairs_of(f);
        }
    } else {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            uint4 w = make_uint4(0u, 0u, 0u, 0u);
            if (k < n) w = reinterpret_cast<const uint4 *>(rows + k * row_bytes)[t];
            float f[8];
            unpack8_bf16(w, f);
            v[k] = pairs_of(f);
        }
    }
}
template <int R, bool ALL>
ECHO_DEV void store_rows(uint8_t *to, int64_t stride, bool f32, const int (&m)[R], const Pairs (&v)[R]) {
#pragma unroll
    for (int k = 0; k < R; ++k, to += stride) {
        float f[8];
        floats_of(v[k], f);
        if (ALL || m[k] >= 0) store8(to, 0, f32, f);
    }
}

// 1 / root of the rows' spread, v centred (LAYER); between(): after the first barrier
template <int R, typename F>
ECHO_DEV void spreads(const Norm &n, float inv_d, bool live, Pairs (&v)[R], float (&f)[R], float4 (*part)[32], int &turn, F between) {
    if (n.kind == ECHO_NORM_LAYER) {
#pragma unroll
        for (int k = 0; k < R; ++k) f[k] = sum8(v[k]);
        block_sums<R>(f, part, turn);
        between();
        const float less = live ? -inv_d : 0.f;      // threads past the row's end keep their zeros
#pragma unroll
        for (int k = 0; k < R; ++k) v[k] = add8(v[k], splat(f[k] * less));
    }
#pragma unroll
    for (int k = 0; k < R; ++k) f[k] = square8(v[k]);
    block_sums<R>(f, part, turn);
    if (n.kind != ECHO_NORM_LAYER) between();
#pragma unroll
    for (int k = 0; k < R; ++k) f[k] = rsqrtf(f[k] * inv_d + n.eps);
}
template <int R, bool AFTER, int THREADS>
__global__ void __launch_bounds__(THREADS)
gated_norm_rows_kernel(const NormParams p, int *err) {
    extern __shared__ __align__(128) uint8_t buf[];
    __shared__ __align__(8) uint64_t full[2];
    __shared__ float4 part[2][32];
    __shared__ int abort_flag;
    const int t = threadIdx.x;
    const bool live = t < p.chunks;
    const uint32_t xb = (uint32_t)p.chunks * (p.xf ? 32u : 16u), yb = p.y ? (uint32_t)p.chunks * (p.yf ? 32u : 16u) : 0u;
    const uint32_t row_bytes = xb + yb;
    if (t == 0) {
        mbar_init(&full[0], 1);
        mbar_init(&full[1], 1);
        abort_flag = 0;
        fence_barrier_init();
    }
    __syncthreads();
    pdl_enter();
    const int first = (int)((int64_t)p.n_rows * blockIdx.x / gridDim.x);
    const int last = (int)((int64_t)p.n_rows * (blockIdx.x + 1) / gridDim.x);
    const int batches = (last - first + R - 1) / R;
    auto fetch = [&](int i) {            // one thread
        const int r0 = first + i * R, n = min(R, last - r0);
        uint8_t *dst = buf + (i & 1) * (R * row_bytes);
        mbar_arrive_expect_tx(&full[i & 1], n * row_bytes);
        for (int k = 0; k < n; ++k, dst += row_bytes) {
            const int64_t r = r0 + k;
            bulk_load_1d(dst, static_cast<const uint8_t *>(p.x) + r * p.ldx * (p.xf ? 4 : 2), xb, &full[i & 1]);
            if (p.y) bulk_load_1d(dst + xb, static_cast<const uint8_t *>(p.y) + r * p.ldy * (p.yf ? 4 : 2), yb, &full[i & 1]);
        }
    };
    if (t == 0) {
        if (batches > 0) fetch(0);
        if (batches > 1) fetch(1);
    }
    // the modulation's row, for the lanes of a batch's rows; -1: the row is left as it is
    const int lane = t & 31;
    auto mod_of = [&](int i) {
        const int r0 = first + i * R, r = r0 + lane;
        int m = 0;
        if (lane >= min(R, last - r0)) return -1;
        if (p.n_mods >= 0) {
            m = p.mod_rows ? p.mod_rows[r] : r / p.rows_per_mod;
            if ((unsigned)m >= (unsigned)p.n_mods) m = -1;
        }
        return m;
    };
    int mod, next, turn = 0, cur = -1, cur_out = -1;
    const Pairs alpha = splat(p.alpha);
    // of the modulations `cur` and `cur_out`, the norms' weights and biases in them (but for a bias of the first)
    Pairs gate = splat(p.beta), scale = splat(1.f), shift = splat(0.f);
    auto take = [&](int m) {
        if (m == cur || m < 0) return;
        cur = m;
        if (!live) return;
        gate = splat(p.beta);
        if (p.gate) gate = mul8(shared_pairs(p.gate, m * p.ldm + 8 * t, p.mf), gate);
        if constexpr (AFTER) {
            if (p.after.weight && !p.after.bias) gate = mul8(shared_pairs(p.after.weight, 8 * t, true), gate);
        }
    };
    auto take_out = [&](int m) {
        if (m == cur_out || m < 0) return;
        cur_out = m;
        if (!live) return;
        scale = splat(1.f);
        if (p.scale) scale = add8(shared_pairs(p.scale, m * p.ldm + 8 * t, p.mf), scale);
        if (p.shift) shift = shared_pairs(p.shift, m * p.ldm + 8 * t, p.mf);
        else shift = splat(0.f);
        if (p.before.bias) shift = fma8(shared_pairs(p.before.bias, 8 * t, true), scale, shift);
        if (p.before.weight) scale = mul8(shared_pairs(p.before.weight, 8 * t, true), scale);
    };
    uint8_t *h_to = static_cast<uint8_t *>(p.h) + (first * p.ldh + 8 * t) * (p.hf ? 4 : 2);
    uint8_t *n_to = static_cast<uint8_t *>(p.n) + (first * p.ldn + 8 * t) * (p.nf ? 4 : 2);
    const int64_t h_row = p.ldh * (p.hf ? 4 : 2), n_row = p.ldn * (p.nf ? 4 : 2);
    next = mod_of(0);
    bool ok = true;
    int i = 0;
    // a batch of rows; SAME: R rows, all of the modulation that is in registers
    auto batch = [&](auto SAME, int n) {
        const uint8_t *rows = buf + (i & 1) * (R * row_bytes);
        auto refill = [&]() {            // the rows are in registers, behind a barrier
            if (t == 0 && ok && i + 2 < batches) fetch(i + 2);
        };
        int m[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            m[k] = 0;
            if constexpr (SAME) continue;
            m[k] = __shfl_sync(0xffffffffu, mod, k);
            if (!ok) m[k] = -1;
        }
        Pairs h[R];
        float f[R];
        const int there = !live ? 0 : SAME ? R : n;
        Pairs one[1];                    // the other of x and y, a row at a time
        if constexpr (AFTER) {
            staged<R>(rows + xb, row_bytes, p.yf, t, there, h);
            spreads<R>(p.after, p.inv_d, live, h, f, part, turn, [] {});
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if constexpr (!SAME) take(m[k]);
                h[k] = mul8(h[k], splat(f[k]));
                if (p.after.bias && live) {
                    if (p.after.weight) h[k] = mul8(h[k], shared_pairs(p.after.weight, 8 * t, true));
                    h[k] = add8(h[k], shared_pairs(p.after.bias, 8 * t, true));
                }
                staged<1>(rows + k * row_bytes, row_bytes, p.xf, t, there - k, one);
                h[k] = fma8(gate, h[k], mul8(one[0], alpha));
            }
        } else {
            staged<R>(rows, row_bytes, p.xf, t, there, h);
#pragma unroll
            for (int k = 0; k < R; ++k) {
                h[k] = mul8(h[k], alpha);
                if (!p.y) continue;
                staged<1>(rows + k * row_bytes + xb, row_bytes, p.yf, t, there - k, one);
                if constexpr (!SAME) take(m[k]);
                h[k] = fma8(gate, one[0], h[k]);
            }
        }
        if (p.h && live) store_rows<R, SAME>(h_to, h_row, p.hf, m, h);
        const bool normed = p.n && p.before.kind != ECHO_NORM_NONE;
        if (normed) {
            spreads<R>(p.before, p.inv_d, live, h, f, part, turn, refill);
        } else {
            __syncthreads();
            refill();
#pragma unroll
            for (int k = 0; k < R; ++k) f[k] = 1.f;
        }
        if (p.n && live) {
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if constexpr (!SAME) take_out(m[k]);
                h[k] = fma8(mul8(h[k], splat(f[k])), scale, shift);
            }
            store_rows<R, SAME>(n_to, n_row, p.nf, m, h);
        }
        if constexpr (!SAME) {
            // as the threads that have columns, whatever was asked for
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (!live || !p.y) take(m[k]);
                if (!live || !p.n) take_out(m[k]);
            }
        }
    };
    for (; i < batches; ++i) {
        const int n = min(R, last - first - i * R);
        mod = next;
        if (i + 1 < batches) next = mod_of(i + 1);
        // a wait that gives up lets the others give up; nothing is stored from then on.  By whole warps:
        // its lanes may have seen different things, and they exchange values below
        ok = __all_sync(0xffffffffu, ok && mbar_wait(&full[i & 1], (i >> 1) & 1, &abort_flag, err));
        // the whole warp takes one way: a barrier lies on both
        if (__all_sync(0xffffffffu, ok && (lane >= R || (mod >= 0 && mod == cur && mod == cur_out)))) batch(std::true_type(), R);
        else batch(std::false_type(), n);
        h_to += R * h_row;
        n_to += R * n_row;
    }
    // copies land before this block exits
    if (!ok && t == 0) {
        for (int i = 0; i < 4; ++i) mbar_land(&full[i & 1], i >> 1);
    }
}

// Few rows: one to a block, a chunk to a thread, and everything that it needs asked for before the first
// sum, since the time is that of one access after the other.
ECHO_DEV Pairs chunk_of(const void *p, int64_t at, bool f32) {
    float f[8];
    if (f32) {
        floats4(ld_once(static_cast<const float *>(p) + at), f);
        floats4(ld_once(static_cast<const float *>(p) + at + 4), f + 4);
    } else {
        unpack8_bf16(ld_once(static_cast<const __nv_bfloat16 *>(p) + at), f);
    }
    return pairs_of(f);
}
__global__ void __launch_bounds__(1024)
gated_norm_row_kernel(const NormParams p) {
    __shared__ float4 part[2][32];
    const int t = threadIdx.x;
    const bool live = t < p.chunks;
    int turn = 0;
    pdl_enter();
    for (int r = blockIdx.x; r < p.n_rows; r += gridDim.x) {
        int m = 0;
        const Pairs none = splat(0.f);
        Pairs h[1] = {none}, y[1] = {none};
        if (live) {
            h[0] = chunk_of(p.x, r * p.ldx + 8 * t, p.xf);
            if (p.y) y[0] = chunk_of(p.y, r * p.ldy + 8 * t, p.yf);
        }
        if (p.n_mods >= 0) {
            m = p.mod_rows ? p.mod_rows[r] : r / p.rows_per_mod;
            if ((unsigned)m >= (unsigned)p.n_mods) continue;
        }
        Pairs gate = splat(p.beta), scale = splat(1.f), shift = none;
        if (live) {
            const int64_t at = m * p.ldm + 8 * t;
            if (p.gate) gate = mul8(shared_pairs(p.gate, at, p.mf), gate);
            if (p.scale) scale = add8(shared_pairs(p.scale, at, p.mf), scale);
            if (p.shift) shift = shared_pairs(p.shift, at, p.mf);
            if (p.before.bias) shift = fma8(shared_pairs(p.before.bias, 8 * t, true), scale, shift);
            if (p.before.weight) scale = mul8(shared_pairs(p.before.weight, 8 * t, true), scale);
        }
        float f[1] = {1.f};
        h[0] = mul8(h[0], splat(p.alpha));
        if (p.y) {
            if (p.after.kind != ECHO_NORM_NONE) {
                spreads<1>(p.after, p.inv_d, live, y, f, part, turn, [] {});
                if (live) {
                    if (p.after.bias) h[0] = fma8(shared_pairs(p.after.bias, 8 * t, true), gate, h[0]);
                    if (p.after.weight) gate = mul8(shared_pairs(p.after.weight, 8 * t, true), gate);
                    h[0] = fma8(mul8(y[0], splat(f[0])), gate, h[0]);
                }
            } else {
                h[0] = fma8(y[0], gate, h[0]);
            }
        }
        const int one[1] = {0};
        if (p.h && live) store_rows<1, true>(static_cast<uint8_t *>(p.h) + (r * p.ldh + 8 * t) * (p.hf ? 4 : 2), 0, p.hf, one, h);
        if (!p.n) continue;
        f[0] = 1.f;
        if (p.before.kind != ECHO_NORM_NONE) spreads<1>(p.before, p.inv_d, live, h, f, part, turn, [] {});
        h[0] = fma8(mul8(h[0], splat(f[0])), scale, shift);
        if (live) store_rows<1, true>(static_cast<uint8_t *>(p.n) + (r * p.ldn + 8 * t) * (p.nf ? 4 : 2), 0, p.nf, one, h);
    }
}

template <int TPR, int CH>
void launch(const NormParams &p, cudaStream_t st) {
    static int per_sm[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    int blocks = 1;
    if (dev >= 0 && dev < 64) {
        if (!per_sm[dev] && cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm[dev], gated_norm_kernel<TPR, CH>,
                                                                          TPR, 0) != cudaSuccess)
            per_sm[dev] = 1;
        blocks = per_sm[dev] > 0 ? per_sm[dev] : 1;
    }
    const int64_t most = (int64_t)echo::num_sms() * blocks;
    const int grid = (int)(p.n_rows < most ? p.n_rows : most);
    echo::launch_chained(gated_norm_kernel<TPR, CH>, dim3(grid), dim3(TPR), 0, st, p);
}

template <int R, bool AFTER, int THREADS>
void launch_rows(const NormParams &p, cudaStream_t st) {
    const int threads = (p.chunks + 31) / 32 * 32;
    const size_t smem = 2ull * R * p.chunks * ((p.xf ? 32 : 16) + (p.y ? (p.yf ? 32 : 16) : 0));
    static int attr_done[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && !attr_done[dev]) {
        cudaFuncSetAttribute(gated_norm_rows_kernel<R, AFTER, THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * kBufferBytes);
        attr_done[dev] = 1;
    }
    int blocks = 1;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, gated_norm_rows_kernel<R, AFTER, THREADS>, threads, smem) != cudaSuccess || blocks < 1)
        blocks = 1;
    const int64_t most = (int64_t)echo::num_sms() * blocks;
    const int grid = (int)(p.n_rows < most ? p.n_rows : most);
    echo::launch_chained(gated_norm_rows_kernel<R, AFTER, THREADS>, dim3(grid), dim3(threads), smem, st, p, echo::device_error_ptr());
}

// Rows of up to 8192 values: up to an SM's worth of them, one to a block; else four at a time where two
// buffers of four rows fit into shared memory, and fewer otherwise.  us for 32760 rows of 5120, bf16 (198
// at the rate of a copy): layer norm 211 (two rows at a time 277, three 249); the root of the mean square, with
// less to do between its loads and stores, 223 three at a time (four 234).  With a norm of y before the layer norm:
// root of the mean square 257, layer norm 283; before the root of the mean square, that of y 231.  fp32 and 16380
// rows 183 (148); 1560 rows 13.8 (9.4: three batches a block, the last one half empty), 48 rows 3.7 (6.1 with the rows
// kernel's copies).  From 5128 columns on one row at a time, since 1024 threads leave few registers: 20000 rows of
// 8192 256 (193; two 321), but rows of 5632 and 6144, which need 704 and 768 threads, take 209 and 213 (133, 145): a bound of
// their own was not tried.  More than 8192: a block to a row, neither copied ahead nor with their modulation kept:
// 10000 rows of 8200 260 (97), of 12288 306 (145), of 16384 412 (193).
void launch_width(const NormParams &p, cudaStream_t st) {
    const int c = p.chunks;
    if (c <= 1024) {
        if (p.n_rows <= echo::num_sms()) {
            echo::launch_chained(gated_norm_row_kernel, dim3(p.n_rows), dim3((c + 31) / 32 * 32), 0, st, p);
            return;
        }
        const bool after = p.y && p.after.kind != ECHO_NORM_NONE;
        const int row_bytes = c * ((p.xf ? 32 : 16) + (p.y ? (p.yf ? 32 : 16) : 0));
        const int most = kBufferBytes / row_bytes;     // rows of a buffer
        if (c > 640) return after ? launch_rows<1, true, 1024>(p, st) : launch_rows<1, false, 1024>(p, st);
        if (after) return most >= 4 ? launch_rows<4, true, 640>(p, st) : launch_rows<2, true, 640>(p, st);
        if (most >= 4 && p.before.kind != ECHO_NORM_RMS) return launch_rows<4, false, 640>(p, st);
        return most >= 3 ? launch_rows<3, false, 640>(p, st) : launch_rows<2, false, 640>(p, st);
    }
    if (c <= 1536) return launch<512, 3>(p, st);
    launch<512, 4>(p, st);
}

echo_status check_norm(const echo_norm &n) {
    if (n.kind < ECHO_NORM_NONE || n.kind > ECHO_NORM_RMS) return ECHO_ERR_INVALID_ARG;
    if (n.kind == ECHO_NORM_NONE) return n.weight || n.bias ? ECHO_ERR_INVALID_ARG : ECHO_OK;
    if (!(n.eps >= 0.f) || n.eps - n.eps != 0.f) return ECHO_ERR_INVALID_ARG;
    return echo::aligned16(n.weight) && echo::aligned16(n.bias) ? ECHO_OK : ECHO_ERR_INVALID_ARG;
}
bool finite(float v) { return v - v == 0.f; }
bool known(echo_dtype t) { return t == ECHO_BF16 || t == ECHO_F32; }

}  // namespace

extern "C" echo_status echo_gated_norm(const echo_gated_norm_plan *plan, const echo_modulation *mod, int32_t n_rows,
                                       const void *x, int64_t ldx, echo_dtype xt, const void *y, int64_t ldy,
                                       echo_dtype yt, void *h, int64_t ldh, echo_dtype ht, void *n, int64_t ldn,
                                       echo_dtype nt, echo_stream_t stream) {
    if (!plan) return ECHO_ERR_INVALID_ARG;
    const int D = plan->D;
    if (D < 8 || D > 16384 || D % 8 || n_rows < 0) return ECHO_ERR_SHAPE;
    if (!known(xt) || !known(ht) || !known(nt) || !known(yt)) return ECHO_ERR_INVALID_ARG;
    echo_status s = check_norm(plan->after);
    if (s == ECHO_OK) s = check_norm(plan->before);
    if (s != ECHO_OK) return s;
    if (!finite(plan->alpha) || !finite(plan->beta)) return ECHO_ERR_INVALID_ARG;
    auto bad_ld = [&](const void *p, int64_t ld) { return p && (ld < D || ld % 8); };
    if (bad_ld(x, ldx) || bad_ld(y, ldy) || bad_ld(h, ldh) || bad_ld(n, ldn)) return ECHO_ERR_SHAPE;
    // rows that go over their inputs: each thread writes what it has read
    auto over = [](const void *a, int64_t lda, echo_dtype ta, const void *b, int64_t ldb, echo_dtype tb) {
        return a && a == b && (lda != ldb || ta != tb);
    };
    if (over(h, ldh, ht, x, ldx, xt) || over(h, ldh, ht, y, ldy, yt) || over(n, ldn, nt, x, ldx, xt) ||
        over(n, ldn, nt, y, ldy, yt))
        return ECHO_ERR_SHAPE;
    if (h && h == n) return ECHO_ERR_INVALID_ARG;
    if (mod) {
        if (!known(mod->t)) return ECHO_ERR_INVALID_ARG;
        if (mod->n_mods < 0 || mod->ld < D || mod->ld % 8 || (!mod->rows && mod->rows_per_mod < 1)) return ECHO_ERR_SHAPE;
        if (!echo::aligned16(mod->gate) || !echo::aligned16(mod->scale) || !echo::aligned16(mod->shift) ||
            (reinterpret_cast<uintptr_t>(mod->rows) & 3u))
            return ECHO_ERR_INVALID_ARG;
    }
    if (n_rows == 0 || (!h && !n)) return ECHO_OK;
    if (!x) return ECHO_ERR_INVALID_ARG;
    if (!echo::aligned16(x) || !echo::aligned16(y) || !echo::aligned16(h) || !echo::aligned16(n))
        return ECHO_ERR_INVALID_ARG;
    if (!echo::device_supported()) return ECHO_ERR_UNSUPPORTED;
    NormParams p = {};
    p.x = x;
    p.y = y;
    p.h = h;
    p.n = n;
    p.ldx = ldx;
    p.ldy = ldy;
    p.ldh = ldh;
    p.ldn = ldn;
    p.xf = xt == ECHO_F32;
    p.yf = yt == ECHO_F32;
    p.hf = ht == ECHO_F32;
    p.nf = nt == ECHO_F32;
    p.after = {plan->after.kind, plan->after.eps, plan->after.weight, plan->after.bias};
    p.before = {plan->before.kind, plan->before.eps, plan->before.weight, plan->before.bias};
    p.alpha = plan->alpha;
    p.beta = plan->beta;
    p.inv_d = 1.f / (float)D;
    p.n_rows = n_rows;
    p.chunks = D / 8;
    p.n_mods = -1;
    if (mod) {
        p.gate = mod->gate;
        p.scale = mod->scale;
        p.shift = mod->shift;
        p.mod_rows = mod->rows;
        p.ldm = mod->ld;
        p.n_mods = mod->n_mods;
        p.rows_per_mod = mod->rows_per_mod;
        p.mf = mod->t == ECHO_F32;
    }
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    echo::LaunchScope ls(ECHO_K_GATED_NORM, n_rows, D, p.n_mods, st);
    launch_width(p, st);
    return echo::last_launch_status();
}
