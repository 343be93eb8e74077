// Rotary positions: the columns of each head turned in pairs by the angle position x
// frequency, for queries and keys in one launch.
//
// (y1, y2) = size (x1 cos a - x2 sin a, x2 cos a + x1 sin a).  A value is read once and
// written once and the time is that of the bytes (32760 rows of 80 heads of 128, bf16, neighbouring
// columns: 197 us, 6.8 TB/s, as a plain copy), if the angles cost little: a frequency is held
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
    int Hq, Hk, key_chunk;        // heads; the first of a row's chunks that are the keys'
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

// neighbouring values of T, read and written at once
template <typename T, int N>
struct Some {
    union {
        typename Raw<N * (int)sizeof(T)>::type raw;
        T v[N];
    };
    ECHO_DEV Some() {}
};
template <typename T>
using Vec = Some<T, 16 / (int)sizeof(T)>;

// the heads of a row's chunk, of the queries or of the keys
template <typename T>
struct Heads {
    const T *src;
    T *dst;
    int n;
    ECHO_DEV Heads(const RotaryParams &p, int r, int chunk) {
        const int kv = chunk >= p.key_chunk, h0 = (chunk - (kv ? p.key_chunk : 0)) * p.per;
        src = static_cast<const T *>(p.in[kv]) + r * p.ld_in[kv] + (int64_t)h0 * p.d;
        dst = static_cast<T *>(p.out[kv]) + r * p.ld_out[kv] + (int64_t)h0 * p.d;
        n = min(p.per, (kv ? p.Hk : p.Hq) - h0);
    }
};

// A row's positions on its axes; false: the row is left as it is
ECHO_DEV bool positions(const RotaryParams &p, int r, int (&at)[4]) {
    at[0] = at[1] = at[2] = at[3] = 0;
    if (p.frame > 0) {
        const int t = p.pos[r];
        at[0] = t / p.frame;
        at[1] = (t - at[0] * p.frame) / p.row;
        at[2] = t - at[0] * p.frame - at[1] * p.row;
        return t >= 0;
    }
    bool in = true;
#pragma unroll
    for (int a = 0; a < 4; ++a)
        if (a < p.axes) {
            at[a] = p.pos[(int64_t)r * p.axes + a];
            in &= at[a] >= 0;
        }
    return in;
}
// size times cosine and sine of a pair's angle; size and 0 for pairs that there are none of
ECHO_DEV void angle(const RotaryParams &p, int pair, bool there, const int (&at)[4], float &c, float &s) {
    const uint64_t turn = there ? __ldg(p.turn + pair) : 0ull;
    const int q = pair < p.end[0] ? at[0] : pair < p.end[1] ? at[1] : pair < p.end[2] ? at[2] : at[3];
    // the fraction of a turn, -1/2 .. 1/2, in half turns
    const int32_t f = (int32_t)((turn * (uint64_t)(uint32_t)q) >> 32);
    sincospif((float)f * 4.656612873077393e-10f, &s, &c);
    c *= p.size;
    s *= p.inverse ? -p.size : p.size;
}

// Pairs of neighbouring columns.  Four blocks of an SM, and two pairs to an instruction: three
// blocks and single pairs took 250 us where this takes 197.  A unit of a head is 16 bytes: W values, W / 2 pairs, or beyond the
// turned ones W columns that are copied.
template <typename T>
__global__ void __launch_bounds__(kThreads, 4)
rotary_pairs_kernel(const RotaryParams p) {
    pdl_enter();
    constexpr int W = 16 / (int)sizeof(T), NP = W / 2;
    const int per_block = kThreads / p.units;         // (row, some heads) of a block
    const int slot = threadIdx.x / p.units, u = threadIdx.x - slot * p.units;
    if (slot >= per_block) return;
    const bool turned = u < p.turned;
    PieceWalk walk(blockIdx.x * per_block + slot, gridDim.x * per_block, p.chunks);
    for (; walk.below(p.n_rows); walk.next()) {
        const int r = (int)walk.row;
        int at[4];
        if (!positions(p, r, at)) continue;
        float c[NP], s[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) angle(p, u * NP + i, turned && u * NP + i < p.pairs, at, c[i], s[i]);
        const Heads<T> hd(p, r, (int)walk.piece);
        const T *src = hd.src + u * W;
        T *dst = hd.dst + u * W;
        if (!turned && src == dst) continue;                  // stays as it is
        for (int h = 0; h < hd.n; h += kAtOnce, src += kAtOnce * p.d, dst += kAtOnce * p.d) {
            Vec<T> x[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k)
                if (h + k < hd.n) x[k].raw = *reinterpret_cast<const uint4 *>(src + k * p.d);
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                if (h + k >= hd.n) continue;
                if (turned) {
#pragma unroll
                    for (int i = 0; i < NP; i += 2) {         // two pairs at once
                        T *v = x[k].v + 2 * i;
                        const uint64_t x1 = f2_pack(value(v[0]), value(v[2])), x2 = f2_pack(value(v[1]), value(v[3]));
                        const uint64_t cc = f2_pack(c[i], c[i + 1]), ss = f2_pack(s[i], s[i + 1]), less = f2_pack(-s[i], -s[i + 1]);
                        float y1[2], y2[2];
                        f2_unpack(f2_fma(x1, cc, f2_mul(x2, less)), y1[0], y1[1]);
                        f2_unpack(f2_fma(x2, cc, f2_mul(x1, ss)), y2[0], y2[1]);
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            if (u * NP + i + e >= p.pairs) continue;
                            put(v[2 * e], y1[e]);
                            put(v[2 * e + 1], y2[e]);
                        }
                    }
                }
                *reinterpret_cast<uint4 *>(dst + k * p.d) = x[k].raw;
            }
        }
    }
}

// Halves: column i and column i + pairs lie apart, and the second may begin anywhere.  A warp
// takes some heads through shared memory, whole stretches in and out, and PW neighbouring pairs (2 where
// that fills the lanes) in between, the next heads on their way meanwhile.  32760 rows of 80 heads of 128,
// bf16, 64 pairs: 222 us, 7 pairs 212; with 16 bytes of either half in a thread's registers 64 pairs
// took 222, but 32 pairs 283 and 7, whose halves are not aligned, 890.
template <typename T, int PW>
__global__ void __launch_bounds__(kThreads)
rotary_halves_kernel(const RotaryParams p) {
    constexpr int kBytes = 1024, NP = 4 / PW;         // bytes of a warp; times 32 PW pairs: 128 at most
    __shared__ __align__(16) uint8_t stage[kThreads / 32][kBytes];
    pdl_enter();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    T *mine = reinterpret_cast<T *>(stage[warp]);
    const int head_bytes = p.d * (int)sizeof(T), at_once = min(kBytes / head_bytes, p.per);
    PieceWalk walk(blockIdx.x * (kThreads / 32) + warp, gridDim.x * (kThreads / 32), p.chunks);
    for (; walk.below(p.n_rows); walk.next()) {
        const int r = (int)walk.row;
        int at[4];
        if (!positions(p, r, at)) continue;
        float c[NP][PW], s[NP][PW];
#pragma unroll
        for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int e = 0; e < PW; ++e) {
                const int pair = PW * (lane + 32 * i) + e;
                if (32 * PW * i < p.pairs) angle(p, pair, pair < p.pairs, at, c[i][e], s[i][e]);
            }
        const Heads<T> hd(p, r, (int)walk.piece);
        const uint8_t *src = reinterpret_cast<const uint8_t *>(hd.src);
        uint8_t *dst = reinterpret_cast<uint8_t *>(hd.dst);
        uint4 next[kBytes / 512];                     // the heads after these are on their way
        auto fetch = [&](const uint8_t *from, int heads) {
#pragma unroll
            for (int i = 0; i < kBytes / 512; ++i)
                if ((lane + 32 * i) * 16 < min(heads, at_once) * head_bytes) next[i] = reinterpret_cast<const uint4 *>(from)[lane + 32 * i];
        };
        fetch(src, hd.n);
        for (int h = 0; h < hd.n; h += at_once, dst += at_once * head_bytes) {
            const int some = min(at_once, hd.n - h), bytes = some * head_bytes;
#pragma unroll
            for (int i = 0; i < kBytes / 512; ++i)
                if ((lane + 32 * i) * 16 < bytes) reinterpret_cast<uint4 *>(mine)[lane + 32 * i] = next[i];
            src += at_once * head_bytes;
            if (h + at_once < hd.n) fetch(src, hd.n - h - at_once);
            __syncwarp();
#pragma unroll 4
            for (int k = 0; k < some; ++k) {
                T *head = mine + k * p.d;
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const int pair = PW * (lane + 32 * i);
                    if (pair >= p.pairs) continue;            // PW divides pairs
                    Some<T, PW> a, b;
                    a.raw = *reinterpret_cast<decltype(a.raw) *>(head + pair);
                    b.raw = *reinterpret_cast<decltype(b.raw) *>(head + pair + p.pairs);
#pragma unroll
                    for (int e = 0; e < PW; ++e) {
                        const float x1 = value(a.v[e]), x2 = value(b.v[e]);
                        put(a.v[e], fmaf(x1, c[i][e], -x2 * s[i][e]));
                        put(b.v[e], fmaf(x2, c[i][e], x1 * s[i][e]));
                    }
                    *reinterpret_cast<decltype(a.raw) *>(head + pair) = a.raw;
                    *reinterpret_cast<decltype(b.raw) *>(head + pair + p.pairs) = b.raw;
                }
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < kBytes / 512; ++i)
                if ((lane + 32 * i) * 16 < bytes)
                    reinterpret_cast<uint4 *>(dst)[lane + 32 * i] = reinterpret_cast<const uint4 *>(mine)[lane + 32 * i];
            __syncwarp();
        }
    }
}

// `lanes` lanes work on some heads of a row: as many heads, up to `most`, as leave work for every SM, since
// their angles are the same
void divide(RotaryParams &p, int lanes, int most) {
    auto chunks = [&](int heads) { return (heads + p.per - 1) / p.per; };
    p.per = most;
    while (p.per > 1 && (int64_t)p.n_rows * (chunks(p.Hq) + chunks(p.Hk)) * lanes < 152ll * 4096) p.per /= 2;
    p.key_chunk = chunks(p.Hq);
    p.chunks = p.key_chunk + chunks(p.Hk);
}
int blocks_of(const RotaryParams &p, int per_block) {
    const int64_t blocks = ((int64_t)p.n_rows * p.chunks + per_block - 1) / per_block;
    return (int)(blocks < 65536 ? blocks : 65536);
}

template <typename T>
void launch(RotaryParams &p, bool halves, bool tail, cudaStream_t st) {
    if (!halves) {
        constexpr int W = 16 / (int)sizeof(T);
        p.turned = (2 * p.pairs + W - 1) / W;
        p.units = tail ? p.d / W : p.turned;
        divide(p, p.units, 8);
        echo::launch_chained(rotary_pairs_kernel<T>, dim3(blocks_of(p, kThreads / p.units)), dim3(kThreads), 0, st, p);
        return;
    }
    divide(p, 32, 16);
    echo::launch_chained(p.pairs % 2 || p.pairs < 64 ? rotary_halves_kernel<T, 1> : rotary_halves_kernel<T, 2>,
                         dim3(blocks_of(p, kThreads / 32)), dim3(kThreads), 0, st, p);
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
    p.Hq = Hq;
    p.Hk = Hk;
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
    echo::LaunchScope ls(ECHO_K_ROTARY, n_rows, ((int64_t)Hq + Hk) * d, 2 * total, st);
    if (t == ECHO_BF16) launch<__nv_bfloat16>(p, plan->layout == ECHO_ROTARY_HALVES, tail, st);
    else launch<float>(p, plan->layout == ECHO_ROTARY_HALVES, tail, st);
    return echo::last_launch_status();
}
