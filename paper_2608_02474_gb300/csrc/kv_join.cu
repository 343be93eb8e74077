// The second launch of an attention call over the paged cache: items that several CTAs did
// in pieces (kv_schedule.cuh) become outputs.
#include <cfloat>

#include "kv_schedule.cuh"

namespace {

// The items that were done in pieces, joined: block (c, .) the one that begins in worker
// c's range and goes on beyond it, a warp per row.  With the pieces' maxima m_i and sums
// l_i: out = sum_i 2^(m_i - m) O_i / sum_i 2^(m_i - m) l_i, in the order of the keys.
constexpr int kJoinRows = 16;

template <int D>
__global__ void __launch_bounds__(32 * kJoinRows)
kv_join_kernel(const KvWork w, const float *__restrict__ ws, __nv_bfloat16 *__restrict__ out, int64_t ldo) {
    __shared__ KvFound found;
    KvWalk walk;
    // before the wait: the kernel ahead passed its own, so the lengths are there
    const bool any = kv_find<32 * kJoinRows, true>(w, blockIdx.x, found, walk);
    pdl_enter();
    if (!any) return;
    const int c = blockIdx.x;
    const int64_t from = walk.at;
    const KvSeq &s = walk.s;
    const int nb = s.blocks(w, walk.ntile);
    if (from >= walk.end || from < walk.start || nb == 0) return;   // not begun here, or nothing in it
    // pieces: worker c + i, i = 0 .. n - 1
    int n = 1;
    const int64_t upto = from + kFixedUnits + nb;
    while (walk.unit_of(c + n) < upto) ++n;
    auto covers = [&](int i, int &kb0, int &kb1) {
        kb0 = i == 0 ? 0 : KvWalk::block_at(walk.unit_of(c + i), from, nb);
        kb1 = KvWalk::block_at(walk.unit_of(c + i + 1), from, nb);
    };
    for (int i = 0; i < 3 && i < n; ++i) {   // stored whole: no other piece has any key
        int kb0, kb1;
        covers(i, kb0, kb1);
        if (kb0 == 0 && kb1 == nb) return;
    }
    const int row = blockIdx.y * kJoinRows + ((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int pr = walk.ntile * w.tile + row;
    if (row >= w.tile || pr >= s.packed) return;
    constexpr int E = D / 32;
    const int64_t stride = (int64_t)2 * w.slot_rows * (D + 2);    // to the next worker's first piece
    const float *one = ws + stride * c + stride / 2, *more = ws + stride * (c + 1);
    auto piece = [&](int i) { return i == 0 ? one : more + stride * (i - 1); };
    float m = -FLT_MAX;
    for (int i = lane; i < n; i += 32) {
        int kb0, kb1;
        covers(i, kb0, kb1);
        if (kb0 < kb1) m = fmaxf(m, piece(i)[w.slot_rows * D + 2 * row]);
    }
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
    float l = 0.f, acc[E] = {};
    for (int i0 = 0; i0 < n; i0 += 32) {
        float f = 0.f, li = 0.f;                                   // of piece i0 + lane
        if (i0 + lane < n) {
            int kb0, kb1;
            covers(i0 + lane, kb0, kb1);
            if (kb0 < kb1) {
                const float2 ml = *reinterpret_cast<const float2 *>(piece(i0 + lane) + w.slot_rows * D + 2 * row);
                f = ex2_approx(ml.x - m);
                li = f * ml.y;
            }
        }
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) li += __shfl_xor_sync(0xffffffffu, li, x);
        l += li;
        const unsigned live = __ballot_sync(0xffffffffu, f != 0.f);   // NaN stays in
        const int most = min(32, n - i0);
#pragma unroll 8
        for (int i = 0; i < most; ++i) {
            const float fi = __shfl_sync(0xffffffffu, f, i);
            if (!(live >> i & 1)) continue;
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
    __nv_bfloat16 *dst = out + (int64_t)(s.row + pr / w.group) * ldo + (walk.nhead * w.group + pr % w.group) * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; e += 2) *reinterpret_cast<uint32_t *>(dst + e) = pack_bf16(acc[e] * inv, acc[e + 1] * inv);
}

}  // namespace

namespace echo {

void launch_kv_join(const KvAttention &a, const KvWork &w, cudaStream_t st) {
    if (!w.split) return;
    const int d = a.pool->d;
    LaunchScope ls(ECHO_K_KV_JOIN, a.batch->n_rows, (int64_t)a.Hq * d, w.workers, st);
    launch_chained(d == 64 ? kv_join_kernel<64> : kv_join_kernel<128>,
                   dim3(w.workers, (w.tile + kJoinRows - 1) / kJoinRows), dim3(32 * kJoinRows), 0, st, w,
                   static_cast<const float *>(a.ws), static_cast<__nv_bfloat16 *>(a.out), a.ldo);
}

}  // namespace echo
