// The second launch of an attention call over the paged cache: items that several CTAs did
// in pieces (kv_schedule.cuh) become outputs.
#include <cfloat>

#include "kv_schedule.cuh"

namespace {

// Blocks (c, .): the item that worker c began and others went on with.  With the pieces'
// maxima m_i and sums l_i: out = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i, m = max_i m_i,
// in the order of the workers.  It waits for memory a few times in a row and does little
// else, so that what counts is how much of an item is on its way at once: R rows of it per
// warp (many rows, few pieces: chunks), or a row's pieces dealt to PARTS warps (few rows,
// many pieces), added up at the end in the order of the parts.
constexpr int kWarps = 8;

template <int D, int R, int PARTS>
__global__ void __launch_bounds__(32 * kWarps)
kv_join_kernel(const KvWork w, float *ws, __nv_bfloat16 *__restrict__ out, int64_t ldo) {
    pdl_enter();
    const KvJoin *joins = kv_joins(ws, w, D) + blockIdx.x;
    constexpr int E = D / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % PARTS;
    // the ends of worker c + 1 + lane, on their way before it is known whether they are needed
    int64_t end = (int)blockIdx.x + lane + 1 < w.workers ? joins[lane].end : INT64_MAX;
    const KvJoin j = *joins;
    const int row0 = (blockIdx.y * (kWarps / PARTS) + warp / PARTS) * R;
    if (j.upto == 0 || (int)blockIdx.y * (kWarps / PARTS) * R >= j.rows) return;
    // pieces: this worker's and those of the workers after it whose units begin before upto
    int n = 1;
    for (int i0 = 0;; i0 += 32) {
        const int i = i0 + lane;
        if (i0 > 0) end = (int)blockIdx.x + i + 1 < w.workers ? joins[i].end : INT64_MAX;
        const int some = __popc(__ballot_sync(0xffffffffu, end < j.upto));
        n += some;
        if (some < 32) break;
    }
    const int64_t slot = (int64_t)w.slot_rows * (D + 2);
    // piece 0 in this worker's second slot, piece i in worker c + i's first
    auto piece = [&](int i) -> const float * { return ws + slot * (2 * (blockIdx.x + i) + (i == 0 ? 1 : 0)); };
    auto ml_of = [&](int i, int r) -> float2 {
        return i < n && row0 + r < j.rows
                   ? *reinterpret_cast<const float2 *>(piece(i) + w.slot_rows * D + 2 * (row0 + r))
                   : make_float2(-FLT_MAX, 0.f);
    };
    float m[R], l[R] = {}, acc[R][E] = {};
#pragma unroll
    for (int r = 0; r < R; ++r) m[r] = -FLT_MAX;
    for (int i0 = 0; i0 < n; i0 += 32)
#pragma unroll
        for (int r = 0; r < R; ++r) m[r] = fmaxf(m[r], ml_of(i0 + lane, r).x);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) m[r] = fmaxf(m[r], __shfl_xor_sync(0xffffffffu, m[r], x));
    for (int i0 = 0; i0 < n; i0 += 32) {
        float f[R];                                        // of piece i0 + lane
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float2 ml = ml_of(i0 + lane, r);
            f[r] = ex2_approx(ml.x - m[r]);
            float li = f[r] * ml.y;
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) li += __shfl_xor_sync(0xffffffffu, li, x);
            l[r] += li;
        }
        const int some = min(32, n - i0);
#pragma unroll 8
        for (int i = part; i < some; i += PARTS) {
            const float *src = piece(i0 + i) + row0 * D + lane * E;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float fi = __shfl_sync(0xffffffffu, f[r], i);
                if (row0 + r >= j.rows) continue;
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    const float2 v = *reinterpret_cast<const float2 *>(src + r * D + e);
                    acc[r][e] += fi * v.x;
                    acc[r][e + 1] += fi * v.y;
                }
            }
        }
    }
    if constexpr (PARTS > 1) {
        __shared__ float sum[kWarps][R * E][32];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int e = 0; e < E; ++e) sum[warp][r * E + e][lane] = acc[r][e];
        __syncthreads();
        if (part > 0) return;
#pragma unroll
        for (int q = 1; q < PARTS; ++q)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int e = 0; e < E; ++e) acc[r][e] += sum[warp + q][r * E + e][lane];
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (row0 + r >= j.rows) continue;
        const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
        const int pr = j.packed0 + row0 + r;
        const int at = w.by_group(pr);
        __nv_bfloat16 *dst = out + (int64_t)(j.row + at) * ldo + (j.head * w.group + pr - at * w.group) * D + lane * E;
#pragma unroll
        for (int e = 0; e < E; e += 2)
            *reinterpret_cast<uint32_t *>(dst + e) = pack_bf16(acc[r][e] * inv, acc[r][e + 1] * inv);
    }
}

template <int R, int PARTS>
void launch(const echo::KvAttention &a, const KvWork &w, cudaStream_t st) {
    constexpr int ROWS = kWarps / PARTS * R;
    echo::launch_chained(a.pool->d == 64 ? kv_join_kernel<64, R, PARTS> : kv_join_kernel<128, R, PARTS>,
                         dim3(w.workers, (w.tile + ROWS - 1) / ROWS), dim3(32 * kWarps), 0, st, w,
                         static_cast<float *>(a.ws), static_cast<__nv_bfloat16 *>(a.out), a.ldo);
}

}  // namespace

namespace echo {

void launch_kv_join(const KvAttention &a, const KvWork &w, cudaStream_t st) {
    if (!w.split) return;
    LaunchScope ls(ECHO_K_KV_JOIN, a.batch->n_rows, (int64_t)a.Hq * a.pool->d, w.workers, st);
    // Few rows: a row's pieces dealt to four warps where there are many of them, or to so many
    // that all rows of all items are in one wave of blocks (128 items in 304 pieces, 32 rows:
    // 25.7 us a call with four warps a row, 22.4 with one; one item in 304 pieces, 24 rows:
    // 36.7, 56.7)
    const int64_t items = (int64_t)a.batch->n_seqs * w.H;
    if (w.tile > kDecodeRows) launch<4, 1>(a, w, st);
    else if (w.tile <= 8 || items * 16 < w.workers) launch<1, 4>(a, w, st);
    else if (w.tile <= 16) launch<1, 2>(a, w, st);
    else launch<1, 1>(a, w, st);
}

}  // namespace echo
