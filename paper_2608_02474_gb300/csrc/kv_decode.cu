// Attention over the paged cache where a sequence has few packed rows (single tokens,
// drafts): 16 at a time, so that the bytes of the pages bound it.
//
// One CTA works through its share of the items (kv_schedule.cuh): a producer warp copies
// key blocks (K and V of one head, and the scales of int8 pages) page by page into a ring
// in shared memory, ahead by whole stages; four warps take a quarter of a block's keys
// each, on m16n8k16 tensor-core products: S = Q K^T, the running maximum and sum of its
// own keys, O += P V.  Nothing passes between the warps until the end of a piece, where
// the four (maximum, sum, O) are joined in a fixed order.
//
// int8 codes become bf16 exactly in registers (kv_codes2).  The keys' scales multiply the scores, the values' scales the weights.
// ldmatrix hands out 16-bit units, so a lane gets neighbouring pairs of codes: Q's columns
// are taken in the same order, and O's columns come out in it.
#include <cfloat>

#include "kv_schedule.cuh"

namespace {

constexpr int WARPS = 4;                       // that compute
constexpr int THREADS = 32 * (WARPS + 1);
constexpr int ROWS = 16;
constexpr int PIECES = 4;                      // handed out ahead

template <bool INT8, int D>
struct Cfg {
    static constexpr int KPW = INT8 ? 32 : 16;             // keys of a warp
    static constexpr int BK = WARPS * KPW;                 // keys of a block
    static constexpr int BSHIFT = INT8 ? 7 : 6;
    static constexpr int ROW_BYTES = INT8 ? D : 2 * D;
    static constexpr int HALF = BK * ROW_BYTES;            // K or V of a block
    static constexpr int SCALES = INT8 ? 2 * BK * 4 : 0;
    static constexpr int STAGE = 2 * HALF + SCALES;        // a multiple of 1024
    static constexpr int JOIN = ROWS * D * 4;              // two warps' half of O
    static constexpr int RING = (110 * 1024 - JOIN) / STAGE;   // two CTAs share an SM
    static constexpr int SMEM = RING * STAGE + JOIN + 1024;
    static_assert(STAGE % 1024 == 0 && RING >= 3, "");
};

struct DecodeParams {
    KvPool pool;
    KvWork work;
    const __nv_bfloat16 *q;
    __nv_bfloat16 *out;
    float *ws;
    int64_t ldq, ldo;
    float scale_log2;
    int *err;
};

ECHO_DEV void ldsm4(uint32_t addr, uint32_t *r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
ECHO_DEV void ldsm4_t(uint32_t addr, uint32_t *r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
ECHO_DEV void mma16816(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// byte offset of 16-byte chunk c of row r of a block's K or V, as the tensor maps lay it out
template <bool INT8, int D>
ECHO_DEV uint32_t chunk_at(int r, int c) {
    if constexpr (INT8 && D == 64) return (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
    else {
        constexpr int BK = Cfg<INT8, D>::BK;
        return (uint32_t)((c >> 3) * (BK * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4));
    }
}

template <bool INT8, int D>
__global__ void __launch_bounds__(THREADS, 2)
kv_decode_kernel(const __grid_constant__ CUtensorMap tm, const DecodeParams p) {
    using C = Cfg<INT8, D>;
    constexpr int KPW = C::KPW, BK = C::BK, NT = KPW / 8, OT = D / 8;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                ~static_cast<uintptr_t>(1023));
    float *join = reinterpret_cast<float *>(smem + C::RING * C::STAGE);
    __shared__ __align__(8) uint64_t full[C::RING], empty[C::RING], piece_full[PIECES], piece_empty[PIECES];
    __shared__ KvPiece piece[PIECES];
    __shared__ float2 row_ml[WARPS][ROWS];
    __shared__ KvFound found;
    __shared__ int abort_flag;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::RING; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], WARPS);
        }
        for (int i = 0; i < PIECES; ++i) {
            mbar_init(&piece_full[i], 1);
            mbar_init(&piece_empty[i], WARPS);
        }
        abort_flag = 0;
        fence_barrier_init();
        tma_prefetch_desc(&tm);
    }
    volatile int *abort_v = &abort_flag;
    pdl_enter();
    KvWalk walk;
    kv_find<THREADS>(p.work, blockIdx.x, found, walk);   // and its barriers

    if (warp == WARPS) {
        // ---------------- producer: the pieces' blocks, a page or part of one at a time ----
        const int shift = p.pool.shift, cs = min(shift, C::BSHIFT);   // tokens of a copy: 1 << cs
        const int per_block = BK >> cs;
        int g = 0;
        bool ok = true, tail = false;
        for (int n = 0; ok; ++n) {
            const bool more = walk.next(p.work);
            if (n >= PIECES) {
                ok = __all_sync(0xffffffffu, mbar_wait(&piece_empty[n % PIECES], ((n / PIECES) & 1) ^ 1, abort_v, p.err));
                if (!ok) break;
            }
            if (lane == 0) {
                KvPiece &pc = piece[n % PIECES];
                if (more) walk.put(p.work, pc);
                else pc.blocks = -1;
                mbar_arrive(&piece_full[n % PIECES]);
                if (more ? walk.tail() : !tail) kv_leave_join(p.work, walk, p.ws, D);
            }
            if (!more) break;
            tail |= walk.tail();
            const int keys = walk.s.keys(p.work, walk.tile);
            if (walk.s.len > p.work.cap) echo_flag_error(p.err, ECHO_ERR_PAGE);
            const int copies = (keys + (1 << cs) - 1) >> cs;
            const int32_t *table = p.work.b.table + (int64_t)walk.seq * p.work.b.max_pages;
            auto page_of = [&](int c) -> int {
                if (c >= copies) return 0;
                const int page = table[(int)(((int64_t)c << cs) >> shift)];
                if ((unsigned)page < (unsigned)p.pool.n_pages) return page;
                echo_flag_error(p.err, ECHO_ERR_PAGE);
                return 0;
            };
            // the pages of 32 copies in the lanes, those of the next 32 on their way
            int c0 = walk.kb0 * per_block;
            int now = page_of(c0 + lane), then = page_of(c0 + 32 + lane);
            for (int kb = walk.kb0; kb < walk.kb1; ++kb, ++g) {
                const int stage = g % C::RING, first = kb * per_block;
                if (first >= c0 + 32) {
                    c0 += 32;
                    now = then;
                    then = page_of(c0 + 32 + lane);
                }
                ok = __all_sync(0xffffffffu, mbar_wait(&empty[stage], ((g / C::RING) & 1) ^ 1, abort_v, p.err));
                if (!ok) break;
                const int n = min(per_block, copies - first);
                if (lane == 0) mbar_arrive_expect_tx(&full[stage], (uint32_t)(n << cs) * (2 * C::ROW_BYTES + (INT8 ? 8 : 0)));
                const int page = __shfl_sync(0xffffffffu, now, (first - c0 + lane) & 31);
                __syncwarp();
                if (lane < n) {
                    uint8_t *dst = smem + stage * C::STAGE;
                    const int y = ((first + lane) << cs) & ((1 << shift) - 1), r0 = lane << cs;
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv) {
                        const int z = (page * 2 + kv) * p.pool.H + walk.head;
                        if constexpr (INT8) {
                            tma_load_3d(dst + kv * C::HALF + r0 * D, &tm, &full[stage], 0, y, z);
                            bulk_load_1d(dst + 2 * C::HALF + (kv * BK + r0) * 4,
                                         p.pool.scale + (((int64_t)z << shift) + y), 4u << cs, &full[stage]);
                        } else {
#pragma unroll
                            for (int a = 0; a < D / 64; ++a)
                                tma_load_3d(dst + kv * C::HALF + a * (BK * 128) + r0 * 128, &tm, &full[stage],
                                            64 * a, y, z);
                        }
                    }
                }
            }
        }
        if (*abort_v && lane == 0)   // let this CTA's copies land before it exits
            for (int i = max(0, g - C::RING); i < g; ++i)
                mbar_wait(&full[i % C::RING], (i / C::RING) & 1, abort_v, nullptr, 100000000ull);
        return;
    }

    // ---------------- four warps, a quarter of each block's keys each ----------------
    const int gq = lane >> 2, tq = lane & 3;        // row group and column pair of a fragment
    const uint32_t ring = smem_u32(smem);
    // lane's row and chunk in a ldmatrix of four 8x8 matrices
    const int mi = lane >> 3, mr = lane & 7;
    int g = 0;
    bool ok = true;
    for (int n = 0; ok; ++n) {
        ok = __all_sync(0xffffffffu, mbar_wait(&piece_full[n % PIECES], (n / PIECES) & 1, abort_v, p.err));
        ok = !named_bar_or(1, 32 * WARPS, !ok);      // the four warps stay together
        const KvPiece &pc = piece[n % PIECES];
        if (!ok || pc.blocks < 0) break;
        KvSeq s;
        s.row = pc.row;
        s.packed = pc.packed;
        s.len = pc.len;
        s.shift = pc.shift;
        const int keys = pc.keys, low = pc.low, group = p.work.group, tile = pc.tile, head = pc.head;
        const int kb0 = pc.kb0, kb1 = kb0 + pc.blocks;
        // rows gq and gq + 8 of the tile: their queries, and the keys that they see
        uint32_t qa[D / 16][4];
        int lim[2];
        int64_t at[2];                               // row and first column of the row's head
        bool real[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int pr = tile * ROWS + gq + 8 * i;
            real[i] = pr < s.packed;
            const int r = s.row + pr / group, h = head * group + pr % group;
            lim[i] = real[i] ? s.top(p.work, r) : keys;
            at[i] = real[i] ? (int64_t)r * p.ldq + h * D : 0;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                uint2 v = make_uint2(0u, 0u);
                if (real[i]) {
                    const __nv_bfloat16 *src = p.q + at[i] + 16 * kk;
                    if constexpr (INT8) {
                        v = *reinterpret_cast<const uint2 *>(src + 4 * tq);
                    } else {
                        v.x = *reinterpret_cast<const uint32_t *>(src + 2 * tq);
                        v.y = *reinterpret_cast<const uint32_t *>(src + 2 * tq + 8);
                    }
                }
                qa[kk][i] = v.x;
                qa[kk][i + 2] = v.y;
            }
        }
        float o[OT][4] = {}, m[2] = {-FLT_MAX, -FLT_MAX}, l[2] = {0.f, 0.f};
        for (int kb = kb0; kb < kb1; ++kb, ++g) {
            const int stage = g % C::RING;
            ok = __all_sync(0xffffffffu, mbar_wait(&full[stage], (g / C::RING) & 1, abort_v, p.err));
            if (!ok) break;
            const int key0 = kb * BK + warp * KPW;       // this warp's first key
            const uint32_t kbase = ring + stage * C::STAGE, vbase = kbase + C::HALF;
            if (key0 < keys) {
                // S = Q K^T
                float sc[NT][4] = {};
                if constexpr (INT8) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int c = 0; c < D / 16; c += 4) {
                            uint32_t r[4];
                            ldsm4(kbase + chunk_at<INT8, D>(warp * KPW + nt * 8 + mr, c + mi), r);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t w = kv_flip(r[i]);
                                mma16816(sc[nt], qa[c + i], kv_codes2(w, 0x4140), kv_codes2(w, 0x4342));
                            }
                        }
                } else {
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
                        for (int nt = 0; nt < NT; nt += 2) {
                            uint32_t r[4];
                            ldsm4(kbase + chunk_at<INT8, D>(warp * KPW + nt * 8 + (mi >> 1) * 8 + mr,
                                                            2 * kk + (mi & 1)), r);
                            mma16816(sc[nt], qa[kk], r[0], r[1]);
                            mma16816(sc[nt + 1], qa[kk], r[2], r[3]);
                        }
                }
                float vs[NT][2];
                const float *scales = reinterpret_cast<const float *>(smem + stage * C::STAGE + 2 * C::HALF);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float2 f = make_float2(p.scale_log2, p.scale_log2);
                    if constexpr (INT8) {
                        const int at2 = warp * KPW + nt * 8 + 2 * tq;
                        const float2 ks = *reinterpret_cast<const float2 *>(scales + at2);
                        const float2 v2 = *reinterpret_cast<const float2 *>(scales + BK + at2);
                        f.x *= ks.x;                 // the codes' unit is in scale_log2
                        f.y *= ks.y;
                        vs[nt][0] = v2.x * kCodeUnit;
                        vs[nt][1] = v2.y * kCodeUnit;
                    }
                    sc[nt][0] *= f.x;
                    sc[nt][1] *= f.y;
                    sc[nt][2] *= f.x;
                    sc[nt][3] *= f.y;
                }
                const bool edge = key0 + KPW > low;      // some row does not see all of these keys
                if (edge) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int j = key0 + nt * 8 + 2 * tq + e;
                            if (INT8 && !(fabsf(vs[nt][e]) < INFINITY)) {   // spoils the rows that see it
                                sc[nt][e] = sc[nt][2 + e] = NAN;
                                vs[nt][e] = 0.f;
                            }
                            if (j >= lim[0]) sc[nt][e] = -INFINITY;
                            if (j >= lim[1]) sc[nt][2 + e] = -INFINITY;
                        }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float mx = -INFINITY;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mx = fmax3(mx, sc[nt][2 * i], sc[nt][2 * i + 1]);
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                    const float m2 = fmaxf(m[i], mx);
                    if (__any_sync(0xffffffffu, m2 > m[i])) {
                        const float a = ex2_approx(m[i] - m2);
                        m[i] = m2;
                        l[i] *= a;
#pragma unroll
                        for (int t = 0; t < OT; ++t) {
                            o[t][2 * i] *= a;
                            o[t][2 * i + 1] *= a;
                        }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float w = ex2_approx(sc[nt][2 * i + e] - m[i]);
                            l[i] += w;
                            sc[nt][2 * i + e] = INT8 ? w * vs[nt][e] : w;
                        }
                }
                // O += P V, 16 keys at a time
                const bool tail = key0 + KPW > keys;     // V rows past the last key: not copied
#pragma unroll
                for (int k2 = 0; k2 < NT / 2; ++k2) {
                    const uint32_t pa[4] = {pack_bf16(sc[2 * k2][0], sc[2 * k2][1]),
                                            pack_bf16(sc[2 * k2][2], sc[2 * k2][3]),
                                            pack_bf16(sc[2 * k2 + 1][0], sc[2 * k2 + 1][1]),
                                            pack_bf16(sc[2 * k2 + 1][2], sc[2 * k2 + 1][3])};
                    const int row = warp * KPW + k2 * 16 + (mi & 1) * 8 + mr;
                    uint32_t keep[2] = {0xffffffffu, 0xffffffffu};
                    if (!INT8 && edge && low < keys) {
                        // rows that do not see all of these keys: values that are not finite
                        // become 0, and spoil the rows that do see them (0 times infinity)
                        uint32_t bad = 0;                    // of the 16 keys
#pragma unroll
                        for (int c = 0; c < C::ROW_BYTES / 16; c += 2) {
                            uint32_t r[4];
                            ldsm4_t(vbase + chunk_at<INT8, D>(row, c + (mi >> 1)), r);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                if ((r[i] & 0x7F80u) == 0x7F80u) bad |= 1u << (8 * (i & 1) + 2 * tq);
                                if ((r[i] & 0x7F800000u) == 0x7F800000u) bad |= 2u << (8 * (i & 1) + 2 * tq);
                            }
                        }
                        bad = __reduce_or_sync(0xffffffffu, bad);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int seen = lim[i] - (key0 + k2 * 16);
                            if (bad & (seen >= 16 ? 0xffffu : seen > 0 ? (1u << seen) - 1u : 0u)) l[i] = NAN;
                            keep[i] = ((bad >> (8 * i + 2 * tq)) & 1 ? 0u : 0xffffu) |
                                      ((bad >> (8 * i + 2 * tq)) & 2 ? 0u : 0xffff0000u);
                        }
                    }
                    if (!INT8 && tail) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int j = key0 + k2 * 16 + 8 * i + 2 * tq;
                            keep[i] &= (j < keys ? 0xffffu : 0u) | (j + 1 < keys ? 0xffff0000u : 0u);
                        }
                    }
#pragma unroll
                    for (int c = 0; c < C::ROW_BYTES / 16; c += 2) {
                        uint32_t r[4];
                        ldsm4_t(vbase + chunk_at<INT8, D>(row, c + (mi >> 1)), r);
                        if constexpr (INT8) {
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const uint32_t w0 = kv_flip(r[2 * i]), w1 = kv_flip(r[2 * i + 1]);
                                mma16816(o[2 * (c + i)], pa, kv_codes2(w0, 0x4240), kv_codes2(w1, 0x4240));
                                mma16816(o[2 * (c + i) + 1], pa, kv_codes2(w0, 0x4341), kv_codes2(w1, 0x4341));
                            }
                        } else {
                            if (edge) {
                                r[0] &= keep[0];
                                r[1] &= keep[1];
                                r[2] &= keep[0];
                                r[3] &= keep[1];
                            }
                            mma16816(o[c], pa, r[0], r[1]);
                            mma16816(o[c + 1], pa, r[2], r[3]);
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[stage]);
        }
        // ---- the four warps' sums, joined in warp order; warp 0 stores ----
        // a wait that gave up is told to all four warps, which leave together
        ok = !named_bar_or(1, 32 * WARPS, !ok);
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
            if (tq == 0) row_ml[warp][gq + 8 * i] = make_float2(m[i], l[i]);
        }
        named_bar_sync(1, 32 * WARPS);
        float mt[2], lt[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            mt[i] = -FLT_MAX;
            lt[i] = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) mt[i] = fmaxf(mt[i], row_ml[w][gq + 8 * i].x);
#pragma unroll
            for (int w = 0; w < WARPS; ++w) {
                const float2 v = row_ml[w][gq + 8 * i];
                lt[i] += ex2_approx(v.x - mt[i]) * v.y;
            }
            const float f = ex2_approx(m[i] - mt[i]);
#pragma unroll
            for (int t = 0; t < OT; ++t) {
                o[t][2 * i] *= f;
                o[t][2 * i + 1] *= f;
            }
        }
        // (0 + 2) + (1 + 3), half the columns at a time through two buffers
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            float *mine = join + (warp & 1) * (OT / 2 * 4 * 32) + lane;
            if (warp >= 2) {
#pragma unroll
                for (int t = 0; t < OT / 2 * 4; ++t) mine[t * 32] = o[hf * OT / 2 + t / 4][t % 4];
            }
            named_bar_sync(1, 32 * WARPS);
            if (warp < 2) {
#pragma unroll
                for (int t = 0; t < OT / 2 * 4; ++t) o[hf * OT / 2 + t / 4][t % 4] += mine[t * 32];
                if (warp == 1) {
#pragma unroll
                    for (int t = 0; t < OT / 2 * 4; ++t) mine[t * 32] = o[hf * OT / 2 + t / 4][t % 4];
                }
            }
            named_bar_sync(1, 32 * WARPS);
            if (warp == 0) {
                const float *other = mine + OT / 2 * 4 * 32;
#pragma unroll
                for (int t = 0; t < OT / 2 * 4; ++t) o[hf * OT / 2 + t / 4][t % 4] += other[t * 32];
            }
            named_bar_sync(1, 32 * WARPS);
        }
        const bool whole = pc.whole;
        float *slot = kv_slot(p.ws, blockIdx.x, pc.tail, ROWS, D);
        __syncwarp();
        if (lane == 0) mbar_arrive(&piece_empty[n % PIECES]);
        if (warp != 0) continue;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (!real[i]) continue;
            const int row = gq + 8 * i, pr = tile * ROWS + row;
            const float inv = lt[i] == 0.f ? 0.f : 1.f / lt[i];      // no key: zeros
            __nv_bfloat16 *dst = p.out + (int64_t)(s.row + pr / group) * p.ldo + (head * group + pr % group) * D;
            float *part = slot + row * D;
            if (!whole && tq == 0) *reinterpret_cast<float2 *>(slot + ROWS * D + 2 * row) = make_float2(mt[i], lt[i]);
            if constexpr (INT8) {
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    const float v[4] = {o[2 * c][2 * i], o[2 * c + 1][2 * i], o[2 * c][2 * i + 1], o[2 * c + 1][2 * i + 1]};
                    if (whole)
                        *reinterpret_cast<uint2 *>(dst + 16 * c + 4 * tq) =
                            make_uint2(pack_bf16(v[0] * inv, v[1] * inv), pack_bf16(v[2] * inv, v[3] * inv));
                    else *reinterpret_cast<float4 *>(part + 16 * c + 4 * tq) = make_float4(v[0], v[1], v[2], v[3]);
                }
            } else {
#pragma unroll
                for (int t = 0; t < OT; ++t) {
                    const float a = o[t][2 * i], b = o[t][2 * i + 1];
                    if (whole) *reinterpret_cast<uint32_t *>(dst + 8 * t + 2 * tq) = pack_bf16(a * inv, b * inv);
                    else *reinterpret_cast<float2 *>(part + 8 * t + 2 * tq) = make_float2(a, b);
                }
            }
        }
    }
}

template <bool INT8, int D>
echo_status launch(const echo::KvAttention &a, cudaStream_t st) {
    using C = Cfg<INT8, D>;
    static int attr_done[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && !attr_done[dev]) {
        cudaFuncSetAttribute(kv_decode_kernel<INT8, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
        attr_done[dev] = 1;
    }
    CUtensorMap tm;
    if (!echo::make_tmap_pages(&tm, *a.pool, (uint32_t)(a.pool->page_tokens < C::BK ? a.pool->page_tokens : C::BK)))
        return ECHO_ERR_CUDA;
    DecodeParams p;
    p.pool = echo::kv_pool(*a.pool);
    p.work = echo::kv_work(a, ROWS, ROWS, C::BSHIFT, 2 * echo::num_sms());
    p.q = static_cast<const __nv_bfloat16 *>(a.q);
    p.out = static_cast<__nv_bfloat16 *>(a.out);
    p.ws = static_cast<float *>(a.ws);
    p.ldq = a.ldq;
    p.ldo = a.ldo;
    p.scale_log2 = 1.4426950408889634f / sqrtf((float)D) * (INT8 ? kCodeUnit : 1.f);
    p.err = echo::device_error_ptr();
    {
        echo::LaunchScope ls(ECHO_K_KV_ATTENTION, a.batch->n_rows, (int64_t)a.Hq * D, a.batch->n_seqs, st);
        echo::launch_chained(kv_decode_kernel<INT8, D>, dim3(p.work.workers), dim3(THREADS), C::SMEM, st, tm, p);
    }
    echo::launch_kv_join(a, p.work, st);
    return echo::last_launch_status();
}

}  // namespace

namespace echo {

size_t kv_decode_workspace(const echo_kv_pool &pool) {
    return kv_workspace_bytes(2 * num_sms(), ROWS, pool.d);
}

echo_status launch_kv_decode(const KvAttention &a, cudaStream_t st) {
    const bool i8 = a.pool->kind == ECHO_CACHE_INT8;
    if (a.pool->d == 64) return i8 ? launch<true, 64>(a, st) : launch<false, 64>(a, st);
    return i8 ? launch<true, 128>(a, st) : launch<false, 128>(a, st);
}

}  // namespace echo
