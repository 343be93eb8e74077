// The end of one branch of a block and the beginning of the next, row by row: the branch's
// output normed, gated and added to the residual stream, the result normed and modulated,
//   h = alpha x + beta gate * N_after(y),   n = N_before(h) * (1 + scale) + shift.
// One pass: a row's x and y are read once into registers, h and n written once, and the time is
// that of those bytes.  Sums are fp32 trees over the row's threads, a mean first and then the
// centred squares.  A thread block takes neighbouring rows, which mostly share their modulation,
// so that gate, scale and shift (for fp32 as many bytes as a row's x, y, h and n, and half as many again)
// come from the L1; the rows themselves pass it by.
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
    if constexpr (TPR > 32) {
        float *at = red[turn & 1];
        ++turn;
        if ((threadIdx.x & 31) == 0) at[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < TPR / 32; ++w) v += at[w];
    }
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

// TPR threads to a row, the whole block but for a warp's rows; CH chunks of 8 values a thread
template <int TPR, int CH>
__global__ void __launch_bounds__(TPR == 32 ? 256 : TPR)
gated_norm_kernel(const NormParams p) {
    pdl_enter();
    __shared__ float red[2][TPR / 32];
    constexpr int RPB = TPR == 32 ? 8 : 1;
    const int t = threadIdx.x % TPR;
    const int64_t workers = (int64_t)gridDim.x * RPB, me = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    const int first = (int)(p.n_rows * me / workers), last = (int)(p.n_rows * (me + 1) / workers);
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

template <int TPR, int CH>
void launch(const NormParams &p, cudaStream_t st) {
    constexpr int RPB = TPR == 32 ? 8 : 1, THREADS = TPR == 32 ? 256 : TPR;
    static int per_sm[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    int blocks = 1;
    if (dev >= 0 && dev < 64) {
        if (!per_sm[dev] && cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm[dev], gated_norm_kernel<TPR, CH>,
                                                                          THREADS, 0) != cudaSuccess)
            per_sm[dev] = 1;
        blocks = per_sm[dev] > 0 ? per_sm[dev] : 1;
    }
    const int64_t all = ((int64_t)p.n_rows + RPB - 1) / RPB, most = (int64_t)echo::num_sms() * blocks;
    const int grid = (int)(all < most ? all : most);
    echo::launch_chained(gated_norm_kernel<TPR, CH>, dim3(grid), dim3(THREADS), 0, st, p);
}

void launch_width(const NormParams &p, cudaStream_t st) {
    const int c = p.chunks;
    if (c <= 32) return launch<32, 1>(p, st);
    if (c <= 64) return launch<32, 2>(p, st);
    if (c <= 128) return launch<32, 4>(p, st);
    if (c <= 256) return launch<128, 2>(p, st);
    if (c <= 384) return launch<128, 3>(p, st);
    if (c <= 512) return launch<128, 4>(p, st);
    if (c <= 640) return launch<128, 5>(p, st);
    if (c <= 768) return launch<256, 3>(p, st);
    if (c <= 1024) return launch<256, 4>(p, st);
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
