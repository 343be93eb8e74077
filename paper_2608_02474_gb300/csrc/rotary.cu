// Rotary positions: the columns of each head turned in pairs by the angle position x
// frequency, for queries and keys in one launch.
//
// (y1, y2) = size (x1 cos a - x2 sin a, x2 cos a + x1 sin a).  A value is read once and
// written once and the time is that of the bytes, if the angles cost little: a frequency is held
// in turns, as a 64-bit fraction, so that position x frequency modulo one turn is an integer
// product whose high part is left over - exact for every position, without fp64 - and a thread
// takes the same columns of several heads, whose angles are the same.
#include "common.cuh"
#include "internal.h"

namespace {

constexpr int kThreads = 256;
constexpr int kAtOnce = 4;        // heads of a thread whose loads are on their way together

struct RotaryParams {
    const uint64_t *turn;
    const int32_t *pos;
    const void *in[2];            // queries, keys
    void *out[2];
    int64_t ld_in[2], ld_out[2];
    int heads, first_key;         // of both; the keys' first
    int n_rows, d, pairs, units, turned, chunks, per;   // units of a head, `turned` of them with pairs; heads a thread
    int axes, end[3];             // pairs before the second, third and fourth axis
    int frame, row;
    float size;
    int inverse;
};

template <int BYTES> struct Raw;
template <> struct Raw<16> { using type = uint4; };
template <> struct Raw<8> { using type = uint2; };
template <> struct Raw<4> { using type = uint32_t; };
template <> struct Raw<2> { using type = uint16_t; };

ECHO_DEV float value(const __nv_bfloat16 &x) { return __bfloat162float(x); }
ECHO_DEV float value(const float &x) { return x; }
ECHO_DEV void put(__nv_bfloat16 &to, float x) { to = __float2bfloat16_rn(x); }
ECHO_DEV void put(float &to, float x) { to = x; }

// W neighbouring values of T, read and written at once
template <typename T, int W>
struct Vec {
    union {
        typename Raw<W * (int)sizeof(T)>::type raw;
        T v[W];
    };
    ECHO_DEV Vec() {}
};

// A unit is W neighbouring columns: W / 2 pairs (PAIRS), or W columns of the first half and the
// same of the second (HALVES); beyond the turned ones, W columns that are copied.
template <typename T, bool HALVES, int W>
__global__ void __launch_bounds__(kThreads)
rotary_kernel(const RotaryParams p) {
    pdl_enter();
    constexpr int NP = HALVES ? W : W / 2;            // pairs of a unit
    const int per_block = kThreads / p.units;         // (row, some heads) of a block
    const int slot = threadIdx.x / p.units, u = threadIdx.x - slot * p.units;
    if (slot >= per_block) return;
    PieceWalk walk(blockIdx.x * per_block + slot, gridDim.x * per_block, p.chunks);
    const bool turned = u < p.turned;
    uint64_t turn[NP];
    int axis[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int pair = u * NP + i;
        turn[i] = turned && pair < p.pairs ? p.turn[pair] : 0ull;
        axis[i] = (pair >= p.end[0]) + (pair >= p.end[1]) + (pair >= p.end[2]);
    }
    for (; walk.below(p.n_rows); walk.next()) {
        const int r = (int)walk.row;
        int at[4] = {0, 0, 0, 0};
        if (p.frame > 0) {
            const int t = p.pos[r];
            at[0] = t / p.frame;
            at[1] = (t - at[0] * p.frame) / p.row;
            at[2] = t - at[0] * p.frame - at[1] * p.row;
            if (t < 0) continue;
        } else {
            bool out = false;
#pragma unroll
            for (int a = 0; a < 4; ++a)
                if (a < p.axes) {
                    at[a] = p.pos[(int64_t)r * p.axes + a];
                    out |= at[a] < 0;
                }
            if (out) continue;
        }
        float c[NP], s[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int q = axis[i] == 0 ? at[0] : axis[i] == 1 ? at[1] : axis[i] == 2 ? at[2] : at[3];
            // the fraction of a turn, -1/2 .. 1/2, in half turns
            const int32_t f = (int32_t)((turn[i] * (uint64_t)(uint32_t)q) >> 32);
            sincospif((float)f * 4.656612873077393e-10f, &s[i], &c[i]);
            c[i] *= p.size;
            s[i] *= p.inverse ? -p.size : p.size;
        }
        const int h0 = (int)walk.piece * p.per, h1 = min(h0 + p.per, p.heads);
        for (int h = h0; h < h1; h += kAtOnce) {
            Vec<T, W> x[kAtOnce][HALVES ? 2 : 1];
            T *dst[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int kv = h + k >= p.first_key, hh = h + k - (kv ? p.first_key : 0);
                const T *src = static_cast<const T *>(p.in[kv]) + r * p.ld_in[kv] + hh * p.d;
                dst[k] = static_cast<T *>(p.out[kv]) + r * p.ld_out[kv] + hh * p.d;
                if (h + k >= h1) dst[k] = nullptr;
                if (!turned && src == dst[k]) dst[k] = nullptr;       // stays as it is
                const int col = HALVES && !turned ? 2 * p.pairs + (u - p.turned) * W : u * W;
                src += col;
                if (!dst[k]) continue;
                dst[k] += col;
                x[k][0].raw = *reinterpret_cast<const decltype(x[k][0].raw) *>(src);
                if (HALVES && turned) x[k][HALVES].raw = *reinterpret_cast<const decltype(x[k][0].raw) *>(src + p.pairs);
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                if (!dst[k]) continue;
                if (turned) {
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        T &e1 = HALVES ? x[k][0].v[i] : x[k][0].v[2 * i], &e2 = HALVES ? x[k][HALVES].v[i] : x[k][0].v[2 * i + 1];
                        if (!HALVES && u * NP + i >= p.pairs) continue;
                        const float x1 = value(e1), x2 = value(e2);
                        put(e1, x1 * c[i] - x2 * s[i]);
                        put(e2, x2 * c[i] + x1 * s[i]);
                    }
                }
                *reinterpret_cast<decltype(x[k][0].raw) *>(dst[k]) = x[k][0].raw;
                if (HALVES && turned) *reinterpret_cast<decltype(x[k][0].raw) *>(dst[k] + p.pairs) = x[k][HALVES].raw;
            }
        }
    }
}

template <typename T, bool HALVES, int W>
void launch(RotaryParams &p, bool tail, cudaStream_t st) {
    p.turned = HALVES ? p.pairs / W : (2 * p.pairs + W - 1) / W;
    p.units = HALVES ? p.turned + (tail ? (p.d - 2 * p.pairs) / W : 0) : tail ? p.d / W : p.turned;
    const int per_block = kThreads / p.units;
    // heads a thread: one angle for many values where there are threads enough
    p.per = 8;
    while (p.per > 1 && (int64_t)p.n_rows * ((p.heads + p.per - 1) / p.per) * p.units < 152ll * 4096) p.per /= 2;
    p.chunks = (p.heads + p.per - 1) / p.per;
    const int64_t blocks = ((int64_t)p.n_rows * p.chunks + per_block - 1) / per_block;
    const int grid = (int)(blocks < 65536 ? blocks : 65536);
    echo::launch_chained(rotary_kernel<T, HALVES, W>, dim3(grid), dim3(kThreads), 0, st, p);
}

template <typename T>
void launch_layout(RotaryParams &p, bool halves, bool tail, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    if (!halves) return launch<T, false, V>(p, tail, st);
    // the second half begins at column `pairs`: as wide as its alignment allows
    if (p.pairs % V == 0) return launch<T, true, V>(p, tail, st);
    if (V == 8 && p.pairs % 4 == 0) return launch<T, true, 4>(p, tail, st);
    if (p.pairs % 2 == 0) return launch<T, true, 2>(p, tail, st);
    launch<T, true, 1>(p, tail, st);
}

}  // namespace

extern "C" echo_status echo_rotary_turns(const echo_rotary_params *q, int32_t axes, const int32_t *axis_pairs,
                                         uint64_t *turn, float *size) {
    if (!q || !axis_pairs || !turn || !size) return ECHO_ERR_INVALID_ARG;
    if (axes < 1 || axes > 4) return ECHO_ERR_SHAPE;
    if (!(q->theta >= 1.0) || !isfinite(q->theta) || !(q->factor >= 1.0) || !isfinite(q->factor))
        return ECHO_ERR_INVALID_ARG;
    if (q->scaling < ECHO_SCALING_NONE || q->scaling > ECHO_SCALING_YARN) return ECHO_ERR_INVALID_ARG;
    if (q->scaling == ECHO_SCALING_YARN &&
        (!(q->original > 0.0) || !isfinite(q->original) || !(q->beta_slow >= 0.0) ||
         !(q->beta_fast > q->beta_slow) || !isfinite(q->beta_fast)))
        return ECHO_ERR_INVALID_ARG;
    int total = 0;
    for (int a = 0; a < axes; ++a) {
        if (axis_pairs[a] < 0 || axis_pairs[a] > 128) return ECHO_ERR_SHAPE;
        total += axis_pairs[a];
    }
    if (total < 1 || total > 128) return ECHO_ERR_SHAPE;
    constexpr double kTurn = 6.283185307179586476925;
    for (int a = 0; a < axes; ++a) {
        const int n = axis_pairs[a];
        const double theta = q->scaling == ECHO_SCALING_NTK && n > 1
                                 ? q->theta * pow(q->factor, (double)n / (n - 1)) : q->theta;
        for (int i = 0; i < n; ++i) {
            double f = pow(theta, -(double)i / n);
            if (q->scaling == ECHO_SCALING_LINEAR) f /= q->factor;
            if (q->scaling == ECHO_SCALING_YARN) {
                const double turns = q->original * f / kTurn;
                double keep = (turns - q->beta_slow) / (q->beta_fast - q->beta_slow);
                keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
                f = f * keep + f / q->factor * (1.0 - keep);
            }
            *turn++ = (uint64_t)(f / kTurn * 18446744073709551616.0);   // f <= 1: below 2^62
        }
    }
    *size = q->scaling == ECHO_SCALING_YARN ? (float)(0.1 * log(q->factor) + 1.0) : 1.f;
    return ECHO_OK;
}

extern "C" echo_status echo_rotary(const echo_rotary_plan *plan, const int32_t *pos, int32_t n_rows, int32_t d,
                                   echo_dtype t, int32_t inverse, const void *q, int64_t ldq, int32_t Hq,
                                   void *q_out, int64_t ldqo, const void *k, int64_t ldk, int32_t Hk,
                                   void *k_out, int64_t ldko, echo_stream_t stream) {
    if (!plan) return ECHO_ERR_INVALID_ARG;
    if (plan->layout != ECHO_ROTARY_PAIRS && plan->layout != ECHO_ROTARY_HALVES) return ECHO_ERR_INVALID_ARG;
    if (t != ECHO_BF16 && t != ECHO_F32) return ECHO_ERR_INVALID_ARG;
    if (!(plan->size == plan->size) || plan->size - plan->size != 0.f) return ECHO_ERR_INVALID_ARG;
    if (plan->axes < 1 || plan->axes > 4 || d < 8 || d > 256 || d % 8) return ECHO_ERR_SHAPE;
    int end[4], total = 0;
    for (int a = 0; a < 4; ++a) {
        if (a < plan->axes) {
            if (plan->axis_pairs[a] < 0 || plan->axis_pairs[a] > d / 2) return ECHO_ERR_SHAPE;
            total += plan->axis_pairs[a];
        }
        end[a] = a + 1 < plan->axes ? total : INT32_MAX;
    }
    if (total < 1 || total > d / 2) return ECHO_ERR_SHAPE;
    if (plan->frame_tokens < 0) return ECHO_ERR_SHAPE;
    if (plan->frame_tokens > 0 && (plan->axes != 3 || plan->row_tokens < 1 || plan->frame_tokens % plan->row_tokens))
        return ECHO_ERR_SHAPE;
    if (n_rows < 0 || Hq < 1 || Hk < 0 || (int64_t)Hq + Hk > (1 << 20)) return ECHO_ERR_SHAPE;
    if (ldq < (int64_t)Hq * d || ldqo < (int64_t)Hq * d || ldq % 8 || ldqo % 8) return ECHO_ERR_SHAPE;
    if (Hk > 0 && (ldk < (int64_t)Hk * d || ldko < (int64_t)Hk * d || ldk % 8 || ldko % 8)) return ECHO_ERR_SHAPE;
    if (q == q_out && ldq != ldqo) return ECHO_ERR_SHAPE;
    if (Hk > 0 && k == k_out && ldk != ldko) return ECHO_ERR_SHAPE;
    if (n_rows == 0) return ECHO_OK;
    if (!q || !q_out || !pos || !plan->turn || (Hk > 0 && (!k || !k_out))) return ECHO_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(pos) & 3u) || (reinterpret_cast<uintptr_t>(plan->turn) & 7u))
        return ECHO_ERR_INVALID_ARG;
    if (!echo::aligned16(q) || !echo::aligned16(q_out)) return ECHO_ERR_INVALID_ARG;
    if (Hk > 0 && (!echo::aligned16(k) || !echo::aligned16(k_out))) return ECHO_ERR_INVALID_ARG;
    if (!echo::device_supported()) return ECHO_ERR_UNSUPPORTED;
    RotaryParams p = {};
    p.turn = plan->turn;
    p.pos = pos;
    p.in[0] = q;
    p.in[1] = k;
    p.out[0] = q_out;
    p.out[1] = k_out;
    p.ld_in[0] = ldq;
    p.ld_in[1] = ldk;
    p.ld_out[0] = ldqo;
    p.ld_out[1] = ldko;
    p.heads = Hq + Hk;
    p.first_key = Hq;
    p.n_rows = n_rows;
    p.d = d;
    p.pairs = total;
    p.axes = plan->axes;
    for (int a = 0; a < 3; ++a) p.end[a] = end[a];
    p.frame = plan->frame_tokens;
    p.row = plan->row_tokens;
    p.size = plan->size;
    p.inverse = inverse != 0;
    const bool tail = 2 * total < d && (q != q_out || (Hk > 0 && k != k_out));
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    echo::LaunchScope ls(ECHO_K_ROTARY, n_rows, (int64_t)p.heads * d, 2 * total, st);
    if (t == ECHO_BF16) launch_layout<__nv_bfloat16>(p, plan->layout == ECHO_ROTARY_HALVES, tail, st);
    else launch_layout<float>(p, plan->layout == ECHO_ROTARY_HALVES, tail, st);
    return echo::last_launch_status();
}
