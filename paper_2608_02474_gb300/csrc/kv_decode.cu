// Attention over the paged cache where a sequence has few packed rows (single tokens,
// drafts): 8, 16, 24 or 32 at a time, so that the bytes of the pages bound it.
//
// One CTA works through its share of the items (kv_schedule.cuh): a producer warp copies
// key blocks (K and V of one head, and the scales of int8 pages) page by page into a ring
// in shared memory, ahead by whole stages; four warps take a quarter of a block's keys
// each, and where the registers allow it two such groups take the blocks in turn.  The
// products run on m16n8k16 tensor instructions with the keys and then the values' columns
// as the 16 rows of A, so that 8 packed rows fill the 8 columns of B:
//   S^T = K Q^T,  P^T = 2^(S^T - m) (rounded to bf16, turned round by movmatrix),
//   O^T += V^T P^T.
// (With the packed rows as A, padded to 16, 48 sequences of up to 8190 int8 keys, 32/8
// heads of 128, took 117 us against 92; one token over 131071 bf16 keys takes 92 both ways.)
// A row's maximum comes from the warp's first block of a piece, and moves only when a
// weight passes 2^64; nothing passes between the warps until the end of a piece, where
// their (maximum, sum, O) are joined in a fixed order.
//
// int8 codes become bf16 exactly in registers (kv_codes2).  The keys' scales multiply the
// scores, the values' scales the weights.  ldmatrix hands out 16-bit units, so a lane gets
// neighbouring pairs of codes: Q's columns are taken in the same order, and O's columns
// come out in it.
//
// 4-bit codes become code / 64 in bf16 (kv_nibbles2), and a code times its group's scale is exact
// in bf16 too, so that keys and values can be multiplied out in registers; for 8 packed rows the
// scores of a group stand apart and take the keys' scale in fp32, with fewer multiplications.
// With a quarter of bf16's bytes it is the instructions beside the products that
// bound it, so: the softmax's scale goes into the exponents' multiply-add; a stage of the ring belongs to one group of warps, whose other group neither waits for it nor frees
// it; the queries of the next piece are fetched while this one's sums are joined; and the warps join behind one
// barrier, all of O in shared memory.  Copies are few, too: 32 tokens' keys and values are one, and their scales
// another (pages of 16 tokens: 16 of them; with four copies for the two, up to 128 tokens each, pages of 16 took 98 us
// and not 77, and one token over 301 keys 9.0 and not 8.1).  48 tokens over up to 8190 keys each, 32/8 heads
// of 128: 71.9 us (80 before these; int8 89.5), 282 MB at
// 5.2 TB/s beside some 18 us that do not grow with the keys: launch, finding the work (2.8), the first copies, the ends of pieces, workers that end unevenly.
#include <cfloat>

#include "kv_schedule.cuh"

namespace {

constexpr int PIECES = 4;                      // handed out ahead
constexpr int kWholeKeys = 768;     // 16 heads of 64, one bf16 token: whole 256 keys 9.2 us, 1024 13.4; divided 11.6, 12.1

// LONG: 256 keys of a block and not 128, for 4-bit heads of 64 over much work (48 tokens of 16 heads over
// up to 8190 keys each 82 us and not 94; but one over 2000 18 and not 14)
template <int FORM, int D, int NR, bool LONG>
struct Cfg {
    static constexpr bool CODES = FORM != kBf16;
    static constexpr int ROWS = 8 * NR;
    static constexpr int GROUPS = NR * D <= (CODES ? 64 : 128) || NR == 1 ? 2 : 1;   // of four warps
    static constexpr int WARPS = 4 * GROUPS, THREADS = 32 * (WARPS + 1);
    static constexpr int KPW = LONG ? 64 : CODES ? 32 : 16;   // keys of a warp
    // 16 keys of them at once; twice 16 of codes, but for 32 rows of 4-bit ones, whose registers do not suffice
    // (8 sequences of 7800 tokens, 16 heads of 64: 43.6 us, so 41.6)
    static constexpr int KG = CODES && !(FORM == kInt4 && NR == 4) ? 2 : 1;
    static constexpr int BK = 4 * KPW;                     // keys of a block
    static constexpr int BSHIFT = KPW == 64 ? 8 : CODES ? 7 : 6;
    static constexpr int ROW_BYTES = kv_bytes(FORM, D);
    static constexpr int HALF = BK * ROW_BYTES;            // K or V of a block
    static constexpr int TOKEN_SCALES = FORM == kInt8 ? 4 : FORM == kInt4 ? D / 16 : 0;   // bytes, of K or V
    static constexpr int SCALES = 2 * BK * TOKEN_SCALES;
    static constexpr int STAGE = 2 * HALF + SCALES;        // a multiple of 1024
    // half of the warps' half of O; 4 bits: all of it
    static constexpr int JOIN = (FORM == kInt4 ? WARPS : WARPS / 4) * ROWS * D * 4;
    static constexpr bool Q_SMEM = (NR * D >= 192 && D == 64) || FORM == kInt4;   // the queries' registers do not suffice
    static constexpr int Q_BUF = ROWS * D * 2, Q_BYTES = Q_SMEM ? (FORM == kInt4 ? 2 : 1) * Q_BUF : 0;   // this piece's and the next
    // two CTAs share an SM.  4 bits: a multiple of the groups, so that a stage is always the same group's
    static constexpr bool OWN = FORM == kInt4;
    static constexpr int RING = (110 * 1024 - JOIN - Q_BYTES) / STAGE / (OWN ? GROUPS : 1) * (OWN ? GROUPS : 1);
    static constexpr int SMEM = RING * STAGE + JOIN + Q_BYTES + 1024;
    static_assert(STAGE % 1024 == 0 && RING >= 2, "");
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
ECHO_DEV uint32_t turn8x8(uint32_t a) {        // an 8x8 matrix of bf16, transposed
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
ECHO_DEV void mma16816(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// neighbouring words of shared memory, read at once
template <int N>
ECHO_DEV void load_words(const uint8_t *from, uint32_t (&to)[N]) {
    if constexpr (N == 4) {
        const uint4 v = *reinterpret_cast<const uint4 *>(from);
        to[0] = v.x;
        to[1] = v.y;
        to[2] = v.z;
        to[3] = v.w;
    } else if constexpr (N == 2) {
        const uint2 v = *reinterpret_cast<const uint2 *>(from);
        to[0] = v.x;
        to[1] = v.y;
    } else {
        to[0] = *reinterpret_cast<const uint32_t *>(from);
    }
}

// byte offset of 16-byte chunk c of row r of a block's K or V, as the tensor maps lay it out
template <int FORM, int D, int BK>
ECHO_DEV uint32_t chunk_at(int r, int c) {
    if constexpr (kv_bytes(FORM, D) == 32) return (uint32_t)(r * 32 + ((c ^ ((r >> 2) & 1)) << 4));
    else if constexpr (kv_bytes(FORM, D) == 64) return (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
    else return (uint32_t)((c >> 3) * (BK * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4));
}

template <int FORM, int D, int NR, bool LONG, bool P16>
__global__ void __launch_bounds__((Cfg<FORM, D, NR, LONG>::THREADS), 2)
kv_decode_kernel(const __grid_constant__ CUtensorMap tm, const __grid_constant__ CUtensorMap tm_scales, const DecodeParams p) {
    using C = Cfg<FORM, D, NR, LONG>;
    constexpr bool INT8 = FORM == kInt8, INT4 = FORM == kInt4, CODES = C::CODES;
    constexpr int KG = C::KG, STEP = 16 * KG, BK = C::BK, MT = D / 16, ROWS = C::ROWS;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                ~static_cast<uintptr_t>(1023));
    float *join = reinterpret_cast<float *>(smem + C::RING * C::STAGE);
    uint2 *q_smem = reinterpret_cast<uint2 *>(smem + C::RING * C::STAGE + C::JOIN);
    __shared__ __align__(8) uint64_t full[C::RING], empty[C::RING], piece_full[PIECES], piece_empty[PIECES];
    __shared__ KvPiece piece[PIECES];
    __shared__ float2 row_ml[C::WARPS][ROWS];
    __shared__ KvFound found;
    __shared__ int abort_flag;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::RING; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], C::OWN ? 4 : C::WARPS);
        }
        for (int i = 0; i < PIECES; ++i) {
            mbar_init(&piece_full[i], 1);
            mbar_init(&piece_empty[i], C::WARPS);
        }
        abort_flag = 0;
        fence_barrier_init();
        tma_prefetch_desc(&tm);
        if (INT4) tma_prefetch_desc(&tm_scales);
    }
    volatile int *abort_v = &abort_flag;
    pdl_enter();
    KvWalk walk;
    kv_find<C::THREADS>(p.work, blockIdx.x, found, walk);   // and its barriers

    if (warp == C::WARPS) {
        // ---------------- producer: the pieces' blocks, a page or part of one at a time ----
        const int shift = p.pool.shift, cs = min(shift, INT4 ? 5 : C::BSHIFT);   // tokens of a copy: 1 << cs
        const int per_block = BK >> cs;
        int g = 0;
        bool ok = true;
        if (lane == 0) kv_leave_join(p.work, walk, p.ws, D);
        for (int n = 0; ok; ++n) {
            const bool more = walk.next(p.work);
            const int keys = more ? walk.s.keys(p.work, walk.tile) : 0;
            if (n >= PIECES) {
                ok = __all_sync(0xffffffffu, mbar_wait(&piece_empty[n % PIECES], ((n / PIECES) & 1) ^ 1, abort_v, p.err));
                if (!ok) break;
            }
            if (lane == 0) {
                KvPiece &pc = piece[n % PIECES];
                if (more) walk.put(p.work, pc);
                else pc.blocks = -1;
                mbar_arrive(&piece_full[n % PIECES]);
                if (more && walk.tail()) kv_leave_join(p.work, walk, p.ws, D);
            }
            if (!more) break;
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
                if (lane == 0) mbar_arrive_expect_tx(&full[stage], (uint32_t)(n << cs) * 2 * (C::ROW_BYTES + C::TOKEN_SCALES));
                const int i = INT8 ? lane >> 1 : lane;       // int8: a lane for keys and one for values
                const int page = __shfl_sync(0xffffffffu, now, (first - c0 + i) & 31);
                __syncwarp();
                if (i < n) {
                    uint8_t *dst = smem + stage * C::STAGE;
                    const int y = ((first + i) << cs) & ((1 << shift) - 1), r0 = i << cs;
                    if constexpr (INT4) {                    // a copy's keys, then its values
                        tma_load_4d(dst + 2 * r0 * C::ROW_BYTES, &tm, &full[stage], 0, y, walk.head, 2 * page);
                        tma_load_3d(dst + 2 * C::HALF + 2 * r0 * C::TOKEN_SCALES, &tm_scales, &full[stage], y * (D / 64),
                                    walk.head, 2 * page);
                    } else if constexpr (INT8) {
                        const int kv = lane & 1, z = (page * 2 + kv) * p.pool.H + walk.head;
                        tma_load_3d(dst + kv * C::HALF + r0 * C::ROW_BYTES, &tm, &full[stage], 0, y, z);
                        bulk_load_1d(dst + 2 * C::HALF + (kv * BK + r0) * C::TOKEN_SCALES,
                                     static_cast<const uint8_t *>(p.pool.scale) + (((int64_t)z << shift) + y) * C::TOKEN_SCALES,
                                     (uint32_t)C::TOKEN_SCALES << cs, &full[stage]);
                    } else {
#pragma unroll
                        for (int kv = 0; kv < 2; ++kv)
#pragma unroll
                            for (int a = 0; a < D / 64; ++a)
                                tma_load_3d(dst + kv * C::HALF + a * (BK * 128) + r0 * 128, &tm, &full[stage], 64 * a, y,
                                            (page * 2 + kv) * p.pool.H + walk.head);
                    }
                }
            }
        }
        // copies land before this CTA exits, whoever gives up, and when
        for (int i = max(0, g - C::RING); i < g; ++i) mbar_land(&full[i % C::RING], (i / C::RING) & 1);
        return;
    }

    // ---------------- groups of four warps, a quarter of each block's keys each ----------------
    // a fragment's row group and column pair; lane's row and chunk in four 8x8 matrices
    const int gq = lane >> 2, tq = lane & 3, mi = lane >> 3, mr = lane & 7;
    const int wk0 = (warp & 3) * C::KPW;             // this warp's first key of a block
    // 4 bits: a copy is 32 tokens' keys and then their values, or twice 16 (P16: pages of 16).  Where the next
    // 16 keys lie, and the values
    constexpr int next16 = P16 ? 32 : 16, values = INT4 ? 48 - next16 : 0;
    const uint32_t ring = smem_u32(smem);
    int g = 0;
    bool ok = true;
    for (int n = 0; ok; ++n) {
        ok = __all_sync(0xffffffffu, mbar_wait(&piece_full[n % PIECES], (n / PIECES) & 1, abort_v, p.err));
        ok = !named_bar_or(1, 32 * C::WARPS, !ok);   // the warps stay together
        const KvPiece &pc = piece[n % PIECES];
        if (!ok || pc.blocks < 0) break;
        KvSeq s;
        s.row = pc.row;
        s.packed = pc.packed;
        s.len = pc.len;
        s.shift = pc.shift;
        const int keys = pc.keys, low = pc.low, group = p.work.group, tile = pc.tile, head = pc.head;
        const int kb0 = pc.kb0, kb1 = kb0 + pc.blocks;
        // B of the first product: 8 packed rows a fragment, row gq of them in this lane
        uint32_t qb[C::Q_SMEM ? 1 : NR][C::Q_SMEM ? 1 : MT][2];
        auto query = [&](const KvPiece &of, int pr, int kk) -> uint2 {
            uint2 v = make_uint2(0u, 0u);
            if (pr < of.packed) {
                const int r = p.work.by_group(pr);
                const __nv_bfloat16 *src = p.q + (int64_t)(of.row + r) * p.ldq + (of.head * group + pr - r * group) * D + 16 * kk;
                if constexpr (INT4) {          // a lane's word of 32 columns: 8 of them, 4 a product
                    v = *reinterpret_cast<const uint2 *>(src - 16 * (kk & 1) + 8 * tq + 4 * (kk & 1));
                } else if constexpr (INT8) {
                    v = *reinterpret_cast<const uint2 *>(src + 4 * tq);
                } else {
                    v.x = *reinterpret_cast<const uint32_t *>(src + 2 * tq);
                    v.y = *reinterpret_cast<const uint32_t *>(src + 2 * tq + 8);
                }
            }
            return v;
        };
        // 4 bits: the fragments that this warp fetches for all
        constexpr int QN = (NR * MT + C::WARPS - 1) / C::WARPS;
        uint2 qn[INT4 ? QN : 1];
        auto fetch_queries = [&](const KvPiece &of) {
#pragma unroll
            for (int i0 = 0; i0 < QN; ++i0) {
                const int i = i0 * C::WARPS + warp;
                if (i < NR * MT) qn[INT4 ? i0 : 0] = query(of, of.tile * ROWS + (i / MT) * 8 + gq, i % MT);
            }
        };
        auto keep_queries = [&](uint2 *to) {
#pragma unroll
            for (int i0 = 0; i0 < QN; ++i0) {
                const int i = i0 * C::WARPS + warp;
                if (i < NR * MT) to[i * 32 + lane] = qn[INT4 ? i0 : 0];
            }
        };
        const uint2 *q_now = q_smem + (INT4 ? (n & 1) * (C::Q_BUF / 8) : 0);
        if constexpr (INT4) {
            if (n == 0) {                            // those of later pieces came meanwhile, below
                fetch_queries(pc);
                keep_queries(q_smem);
                named_bar_sync(1, 32 * C::WARPS);
            }
        } else if constexpr (C::Q_SMEM) {            // the fragments as they are, lane by lane
#pragma unroll
            for (int i0 = 0; i0 < NR * MT; i0 += C::WARPS) {
                const int i = i0 + warp;             // WARPS divides NR * MT
                q_smem[i * 32 + lane] = query(pc, tile * ROWS + (i / MT) * 8 + gq, i % MT);
            }
            named_bar_sync(1, 32 * C::WARPS);
        } else {
#pragma unroll
            for (int nt = 0; nt < NR; ++nt)
#pragma unroll
                for (int kk = 0; kk < MT; ++kk) {
                    const uint2 v = query(pc, tile * ROWS + nt * 8 + gq, kk);
                    qb[nt][kk][0] = v.x;
                    qb[nt][kk][1] = v.y;
                }
        }
        // rows 8 nt + 2 tq + e of the tile, in S^T's and O^T's columns: the keys that they see
        int lim[NR][2];
#pragma unroll
        for (int nt = 0; nt < NR; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int pr = tile * ROWS + nt * 8 + 2 * tq + e;
                lim[nt][e] = pr < s.packed ? s.top(p.work, s.row + p.work.by_group(pr)) : keys;
            }
        float o[NR][MT][4] = {}, m[NR][2], l[NR][2];
#pragma unroll
        for (int nt = 0; nt < NR; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) m[nt][e] = -FLT_MAX, l[nt][e] = 0.f;
        bool fresh = true;                           // no maximum yet
        for (int kb = kb0; kb < kb1; ++kb, ++g) {
            // every warp sees every stage fill, its own or not, before the stage is filled again:
            // a barrier's phases are told apart by their parity only
            const bool own = C::GROUPS == 1 || (g & 1) == warp >> 2;
            if (C::OWN && !own) continue;
            const int stage = g % C::RING;
            ok = __all_sync(0xffffffffu, mbar_wait(&full[stage], (g / C::RING) & 1, abort_v, p.err));
            if (!ok) break;
            const uint32_t kbase = ring + stage * C::STAGE, vbase = INT4 ? kbase : kbase + C::HALF;
            if (own)
#pragma unroll 1
            for (int k0 = 0; k0 < C::KPW; k0 += STEP) {
                const int wk = wk0 + k0, key0 = kb * BK + wk;    // the first key of this step, and where it lies
                const int at0 = INT4 ? 2 * (wk & ~31) + (wk & 16 ? next16 : 0) : wk;
                if (key0 >= keys) break;
                // S^T = K Q^T, 16 keys at a time
                float sc[KG][NR][4] = {};
                const uint8_t *token_scales = smem + stage * C::STAGE + 2 * C::HALF;
                constexpr int STEPS = INT4 ? 4 : INT8 ? 2 : 1;   // products of what four matrices hold
                if constexpr (INT4) {
                    // 8 packed rows: a group's scores by themselves, times the keys' scales; more rows: the
                    // scales go into the keys
                    constexpr bool APART = NR == 1;
#pragma unroll
                    for (int kk = 0; kk < MT; kk += STEPS) {
                        uint2 qf[NR][STEPS];
#pragma unroll
                        for (int nt = 0; nt < NR; ++nt)
#pragma unroll
                            for (int i = 0; i < STEPS; ++i) {
                                qf[nt][i] = q_now[(nt * MT + kk + i) * 32 + lane];
                            }
#pragma unroll
                        for (int kg = 0; kg < KG; ++kg) {
                            uint32_t r[4], ks[2];    // two groups' codes; scales of keys gq and gq + 8
                            const int row = at0 + kg * next16 + (mi & 1) * 8 + mr;
                            ldsm4(kbase + chunk_at<FORM, D, BK>(row, kk / 2 + (mi >> 1)), r);
#pragma unroll
                            for (int h = 0; h < 2; ++h)
                                ks[h] = *reinterpret_cast<const uint32_t *>(token_scales + (at0 + kg * next16 + 8 * h + gq) * C::TOKEN_SCALES + kk);
#pragma unroll
                            for (int i = 0; i < 2; ++i) {        // a group of 32 columns
                                uint32_t a[4], c[4];
                                a[0] = kv_nibbles2<0>(r[2 * i]);
                                a[1] = kv_nibbles2<0>(r[2 * i + 1]);
                                a[2] = kv_nibbles2<1>(r[2 * i]);
                                a[3] = kv_nibbles2<1>(r[2 * i + 1]);
                                c[0] = kv_nibbles2<2>(r[2 * i]);
                                c[1] = kv_nibbles2<2>(r[2 * i + 1]);
                                c[2] = kv_nibbles2<3>(r[2 * i]);
                                c[3] = kv_nibbles2<3>(r[2 * i + 1]);
                                if constexpr (APART) {
                                    float part[4] = {};
                                    mma16816(part, a, qf[0][2 * i].x, qf[0][2 * i].y);
                                    mma16816(part, c, qf[0][2 * i + 1].x, qf[0][2 * i + 1].y);
#pragma unroll
                                    for (int e = 0; e < 4; ++e)
                                        sc[kg][0][e] = fmaf(part[e], i ? bf16hi(ks[e / 2]) : bf16lo(ks[e / 2]), sc[kg][0][e]);
                                } else {
                                    const uint32_t both = i ? 0x3232u : 0x1010u;
                                    const uint32_t s0 = __byte_perm(ks[0], 0u, both), s1 = __byte_perm(ks[1], 0u, both);
#pragma unroll
                                    for (int e = 0; e < 4; ++e) {
                                        a[e] = bf16x2_mul(a[e], e & 1 ? s1 : s0);
                                        c[e] = bf16x2_mul(c[e], e & 1 ? s1 : s0);
                                    }
#pragma unroll
                                    for (int nt = 0; nt < NR; ++nt) {
                                        mma16816(sc[kg][nt], a, qf[nt][2 * i].x, qf[nt][2 * i].y);
                                        mma16816(sc[kg][nt], c, qf[nt][2 * i + 1].x, qf[nt][2 * i + 1].y);
                                    }
                                }
                            }
                        }
                    }
                } else {
#pragma unroll
                for (int kg = 0; kg < KG; ++kg)
#pragma unroll
                    for (int kk = 0; kk < MT; kk += STEPS) {
                        uint32_t r[4];
                        const int row = wk + kg * 16 + (mi & 1) * 8 + mr;
                        ldsm4(kbase + chunk_at<FORM, D, BK>(row, INT8 ? kk + (mi >> 1) : 2 * kk + (mi >> 1)), r);
#pragma unroll
                        for (int i = 0; i < STEPS; ++i) {
                            uint32_t a[4] = {r[0], r[1], r[2], r[3]};
                            if constexpr (INT8) {
                                const uint32_t w0 = kv_flip(r[2 * i]), w1 = kv_flip(r[2 * i + 1]);
                                a[0] = kv_codes2(w0, 0x4140);
                                a[1] = kv_codes2(w1, 0x4140);
                                a[2] = kv_codes2(w0, 0x4342);
                                a[3] = kv_codes2(w1, 0x4342);
                            }
#pragma unroll
                            for (int nt = 0; nt < NR; ++nt) {
                                if constexpr (C::Q_SMEM) {
                                    const uint2 b = q_smem[(nt * MT + kk + i) * 32 + lane];
                                    mma16816(sc[kg][nt], a, b.x, b.y);
                                } else {
                                    mma16816(sc[kg][nt], a, qb[nt][kk + i][0], qb[nt][kk + i][1]);
                                }
                            }
                        }
                    }
                }
                // in the exponent of two: keys gq and gq + 8 of each 16, rows 2 tq and 2 tq + 1
                const float *scales = reinterpret_cast<const float *>(token_scales) + wk + gq;
                const bool edge = key0 + STEP > low;      // some row does not see all of these keys
                uint32_t spoilt = 0;                     // 4 bits: of this lane's key, and of all
                if (INT4 && edge) {
                    // values' scales that are not finite, or anything past the end: 0, and what is
                    // spoilt spoils the rows that see it.  This warp's keys alone.
                    uint32_t *at = reinterpret_cast<uint32_t *>(smem + stage * C::STAGE + 2 * C::HALF + (at0 + values + (lane >> 4) * next16 + (lane & 15)) * C::TOKEN_SCALES);
#pragma unroll
                    for (int i = 0; i < (lane < STEP ? C::TOKEN_SCALES / 4 : 0); ++i) {
                        const uint32_t off = kv_not_finite2(at[i]);
                        spoilt |= off;
                        if (off) at[i] &= ~off;
                    }
                    spoilt = __ballot_sync(0xffffffffu, spoilt != 0u);
                    fence_proxy_async_smem();            // before the copies of a later block
                    __syncwarp();
                }
                float vs[KG][2];
#pragma unroll
                for (int kg = 0; kg < KG; ++kg)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float f = p.scale_log2;
                        if constexpr (INT8) {
                            f *= scales[kg * 16 + 8 * h];   // the codes' unit is in scale_log2
                            vs[kg][h] = scales[BK + kg * 16 + 8 * h] * kCodeUnit;
                        }
#pragma unroll
                        for (int nt = 0; nt < NR; ++nt) {
                            if constexpr (INT4) continue;        // below
                            sc[kg][nt][2 * h] *= f;
                            sc[kg][nt][2 * h + 1] *= f;
                        }
                        if (edge) {
                            const int j = key0 + kg * 16 + 8 * h + gq;
                            bool bad = false;        // a value's scale is not finite: it spoils the rows that see it
                            if constexpr (INT8) {
                                bad = !(fabsf(vs[kg][h]) < INFINITY);
                                if (bad) vs[kg][h] = 0.f;
                            }
                            if constexpr (INT4) bad = (spoilt >> (kg * 16 + 8 * h + gq)) & 1u;
#pragma unroll
                            for (int nt = 0; nt < NR; ++nt)
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    float &x = sc[kg][nt][2 * h + e];
                                    if (bad) x = NAN;
                                    if (j >= lim[nt][e]) x = -INFINITY;
                                }
                        }
                    }
                // the rows' maxima over this warp's keys
                auto raise = [&]() {
#pragma unroll
                    for (int nt = 0; nt < NR; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float mx = -INFINITY;
#pragma unroll
                            for (int kg = 0; kg < KG; ++kg) mx = fmax3(mx, sc[kg][nt][e], sc[kg][nt][2 + e]);
#pragma unroll
                            for (int x = 4; x < 32; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
                            if constexpr (INT4) mx *= p.scale_log2;
                            const float m2 = fmaxf(m[nt][e], mx), a = ex2_approx(m[nt][e] - m2);
                            m[nt][e] = m2;
                            l[nt][e] *= a;
#pragma unroll
                            for (int t = 0; t < MT; ++t) {
                                o[nt][t][e] *= a;
                                o[nt][t][2 + e] *= a;
                            }
                        }
                };
                // P^T in fragments of B; the largest weight, NaN included
                uint32_t pb[KG][NR][2];
                float add[NR][2];
                auto weights = [&]() -> bool {
                    bool high = false;
#pragma unroll
                    for (int nt = 0; nt < NR; ++nt) {
                        add[nt][0] = add[nt][1] = 0.f;
#pragma unroll
                        for (int kg = 0; kg < KG; ++kg)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                float w0 = ex2_approx(INT4 ? fmaf(sc[kg][nt][2 * h], p.scale_log2, -m[nt][0]) : sc[kg][nt][2 * h] - m[nt][0]);
                                float w1 = ex2_approx(INT4 ? fmaf(sc[kg][nt][2 * h + 1], p.scale_log2, -m[nt][1])
                                                           : sc[kg][nt][2 * h + 1] - m[nt][1]);
                                add[nt][0] += w0;
                                add[nt][1] += w1;
                                if constexpr (INT8) w0 *= vs[kg][h], w1 *= vs[kg][h];
                                pb[kg][nt][h] = pack_bf16(w0, w1);
                            }
                        high |= !(add[nt][0] <= 1.8446744e19f) || !(add[nt][1] <= 1.8446744e19f);
                    }
                    return __any_sync(0xffffffffu, high);
                };
                if (fresh) raise();
                fresh = false;
                if (weights()) {
                    raise();
                    weights();
                }
#pragma unroll
                for (int nt = 0; nt < NR; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) l[nt][e] += add[nt][e];
                // O^T += V^T P^T
                const bool tail = key0 + STEP > keys;     // V rows past the last key: not copied
#pragma unroll
                for (int kg = 0; kg < KG; ++kg) {
                    uint32_t b[NR][2];
#pragma unroll
                    for (int nt = 0; nt < NR; ++nt) {
                        b[nt][0] = turn8x8(pb[kg][nt][0]);
                        b[nt][1] = turn8x8(pb[kg][nt][1]);
                    }
                    // a matrix of 8 keys and 16 bytes: bf16 keys, then columns; codes the other way
                    const int row = at0 + values + kg * next16 + (CODES ? (mi & 1) : (mi >> 1)) * 8 + mr;
                    const int col = CODES ? mi >> 1 : mi & 1;
                    uint32_t keep[2] = {0xffffffffu, 0xffffffffu};
                    if (!CODES && edge && low < keys) {
                        // rows that do not see all of these keys: values that are not finite
                        // become 0, and spoil the rows that do see them (0 times infinity)
                        uint32_t bad = 0;                    // of the 16 keys
#pragma unroll
                        for (int t = 0; t < MT; ++t) {
                            uint32_t r[4];
                            ldsm4_t(vbase + chunk_at<FORM, D, BK>(row, 2 * t + col), r);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                if ((r[i] & 0x7F80u) == 0x7F80u) bad |= 1u << (8 * (i >> 1) + 2 * tq);
                                if ((r[i] & 0x7F800000u) == 0x7F800000u) bad |= 2u << (8 * (i >> 1) + 2 * tq);
                            }
                        }
                        bad = __reduce_or_sync(0xffffffffu, bad);
#pragma unroll
                        for (int nt = 0; nt < NR; ++nt)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const int seen = lim[nt][e] - (key0 + kg * 16);
                                if (bad & (seen >= 16 ? 0xffffu : seen > 0 ? (1u << seen) - 1u : 0u)) l[nt][e] = NAN;
                            }
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            keep[h] = ((bad >> (8 * h + 2 * tq)) & 1 ? 0u : 0xffffu) |
                                      ((bad >> (8 * h + 2 * tq)) & 2 ? 0u : 0xffff0000u);
                    }
                    if (!CODES && tail) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int j = key0 + kg * 16 + 8 * h + 2 * tq;
                            keep[h] &= (j < keys ? 0xffffu : 0u) | (j + 1 < keys ? 0xffff0000u : 0u);
                        }
                    }
                    // 4 bits: the scales of keys 2 tq, 2 tq + 1 and of 8 keys further on, as the weights lie
                    uint32_t vw[2][2 * (D / 64)];
                    if constexpr (INT4) {
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            load_words(token_scales + (at0 + values + kg * next16 + 8 * h + 2 * tq) * C::TOKEN_SCALES, vw[h]);
                    }
#pragma unroll
                    for (int t = 0; t < MT; t += STEPS) {
                        uint32_t r[4];
                        ldsm4_t(vbase + chunk_at<FORM, D, BK>(row, INT4 ? t / 2 + col : INT8 ? t + col : 2 * t + col), r);
                        if constexpr (INT4) {
#pragma unroll
                            for (int i = 0; i < 2; ++i) {            // a group of 32 columns
                                uint32_t s2[2];
#pragma unroll
                                for (int h = 0; h < 2; ++h)
                                    s2[h] = __byte_perm(vw[h][t / 4], vw[h][D / 64 + t / 4], i ? 0x7632u : 0x5410u);
                                const uint32_t a[4] = {kv_nibbles2<0>(r[2 * i], s2[0]), kv_nibbles2<1>(r[2 * i], s2[0]),
                                                       kv_nibbles2<0>(r[2 * i + 1], s2[1]), kv_nibbles2<1>(r[2 * i + 1], s2[1])};
                                const uint32_t c[4] = {kv_nibbles2<2>(r[2 * i], s2[0]), kv_nibbles2<3>(r[2 * i], s2[0]),
                                                       kv_nibbles2<2>(r[2 * i + 1], s2[1]), kv_nibbles2<3>(r[2 * i + 1], s2[1])};
#pragma unroll
                                for (int nt = 0; nt < NR; ++nt) {
                                    mma16816(o[nt][t + 2 * i], a, b[nt][0], b[nt][1]);
                                    mma16816(o[nt][t + 2 * i + 1], c, b[nt][0], b[nt][1]);
                                }
                            }
                        } else if constexpr (INT8) {
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const uint32_t w0 = kv_flip(r[2 * i]), w1 = kv_flip(r[2 * i + 1]);
                                const uint32_t a[4] = {kv_codes2(w0, 0x4240), kv_codes2(w0, 0x4341),
                                                       kv_codes2(w1, 0x4240), kv_codes2(w1, 0x4341)};
#pragma unroll
                                for (int nt = 0; nt < NR; ++nt) mma16816(o[nt][t + i], a, b[nt][0], b[nt][1]);
                            }
                        } else {
                            if (edge) {
                                r[0] &= keep[0];
                                r[1] &= keep[0];
                                r[2] &= keep[1];
                                r[3] &= keep[1];
                            }
#pragma unroll
                            for (int nt = 0; nt < NR; ++nt) mma16816(o[nt][t], r, b[nt][0], b[nt][1]);
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[stage]);
        }
        // ---- the warps' sums, joined in a fixed order; warp 0 stores ----
        // a wait that gave up is told to all warps, which leave together
        ok = !named_bar_or(1, 32 * C::WARPS, !ok);
        if (!ok) break;
        bool more = false;                           // 4 bits: the next piece's queries on their way
        if constexpr (INT4) {
            const KvPiece &after = piece[(n + 1) % PIECES];
            more = __all_sync(0xffffffffu, mbar_wait(&piece_full[(n + 1) % PIECES], ((n + 1) / PIECES) & 1, abort_v, p.err)) &&
                   after.blocks >= 0;
            if (more) fetch_queries(after);
        }
#pragma unroll
        for (int nt = 0; nt < NR; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], x);
                if constexpr (INT4) l[nt][e] *= 1.f / kNibbleUnit;   // as the values in O
                if (gq == 0) row_ml[warp][nt * 8 + 2 * tq + e] = make_float2(m[nt][e], l[nt][e]);
            }
        named_bar_sync(1, 32 * C::WARPS);
        float mt[NR][2], lt[NR][2];
#pragma unroll
        for (int nt = 0; nt < NR; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                mt[nt][e] = -FLT_MAX;
                lt[nt][e] = 0.f;
#pragma unroll
                for (int w = 0; w < C::WARPS; ++w) mt[nt][e] = fmaxf(mt[nt][e], row_ml[w][nt * 8 + 2 * tq + e].x);
#pragma unroll
                for (int w = 0; w < C::WARPS; ++w) {
                    const float2 v = row_ml[w][nt * 8 + 2 * tq + e];
                    lt[nt][e] += ex2_approx(v.x - mt[nt][e]) * v.y;
                }
                const float f = ex2_approx(m[nt][e] - mt[nt][e]);
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    o[nt][t][e] *= f;
                    o[nt][t][2 + e] *= f;
                }
            }
        float *const flat = &o[0][0][0];
        if constexpr (INT4) {
            // every warp puts down what it has, and adds up the warps' pairs of an even share: one barrier
            constexpr int N = NR * MT * 4, PAIRS = N / 2 / C::WARPS;
            static_assert(MT * 2 % C::WARPS == 0, "a share's pairs are of known rows");
#pragma unroll
            for (int i = 0; i < N; ++i) join[(warp * N + i) * 32 + lane] = flat[i];
            if (more) keep_queries(q_smem + ((n + 1) & 1) * (C::Q_BUF / 8));
            named_bar_sync(1, 32 * C::WARPS);
            const bool whole = pc.whole;
            float *slot = kv_slot(p.ws, blockIdx.x, pc.tail, ROWS, D);
            if (!whole && warp == 0 && gq == 0) {
#pragma unroll
                for (int nt = 0; nt < NR; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int row = nt * 8 + 2 * tq + e;
                        if (tile * ROWS + row < s.packed)
                            *reinterpret_cast<float2 *>(slot + ROWS * D + 2 * row) = make_float2(mt[nt][e], lt[nt][e]);
                    }
            }
#pragma unroll
            for (int k = 0; k < PAIRS; ++k) {
                const int i = k * C::WARPS + warp, nt = k * C::WARPS / (MT * 2);   // pair i: of tile t, column of gq u
                const int t = i / 2 % MT, u = i & 1;
                float x[2] = {0.f, 0.f};
#pragma unroll
                for (int w = 0; w < C::WARPS; ++w)
#pragma unroll
                    for (int e = 0; e < 2; ++e) x[e] += join[(w * N + 2 * i + e) * 32 + lane];
#pragma unroll
                for (int e = 0; e < 2; ++e) x[e] *= !whole ? 1.f : lt[nt][e] == 0.f ? 0.f : 1.f / lt[nt][e];   // no key: zeros
                // columns in pairs, those of lanes gq and gq + 1: even lanes trade row 2 tq + 1 for row 2 tq.
                // They are 8 (gq / 2) + gq mod 2 of each 32, plus 4 (t mod 2), and 2 u
                const int e = gq & 1;
                const float got = __shfl_xor_sync(0xffffffffu, e ? x[0] : x[1], 4);
                const float a = e ? got : x[0], b = e ? x[1] : got;
                const int row = nt * 8 + 2 * tq + e, pr = tile * ROWS + row;
                const int col = 32 * (t >> 1) + 8 * (gq >> 1) + 4 * (t & 1) + 2 * u;
                if (pr < s.packed) {
                    const int r = p.work.by_group(pr);
                    if (whole)
                        *reinterpret_cast<uint32_t *>(p.out + (int64_t)(s.row + r) * p.ldo +
                                                      (head * group + pr - r * group) * D + col) = pack_bf16(a, b);
                    else *reinterpret_cast<float2 *>(slot + row * D + col) = make_float2(a, b);
                }
                __syncwarp();
            }
            if (lane == 0) mbar_arrive(&piece_empty[n % PIECES]);
            continue;
        }
        // warp w takes over warp w + W/2, W/4, ...: half the columns at a time
        constexpr int HALF_O = NR * MT * 2;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
#pragma unroll
            for (int k = C::WARPS / 2; k >= 1; k >>= 1) {
                float *at = join + (warp & (k - 1)) * (HALF_O * 32) + lane;
                if (warp >= k && warp < 2 * k) {
#pragma unroll
                    for (int i = 0; i < HALF_O; ++i) at[i * 32] = flat[hf * HALF_O + i];
                }
                named_bar_sync(1, 32 * C::WARPS);
                if (warp < k) {
#pragma unroll
                    for (int i = 0; i < HALF_O; ++i) flat[hf * HALF_O + i] += at[i * 32];
                }
                named_bar_sync(1, 32 * C::WARPS);
            }
        }
        const bool whole = pc.whole;
        float *slot = kv_slot(p.ws, blockIdx.x, pc.tail, ROWS, D);
        __syncwarp();
        if (lane == 0) mbar_arrive(&piece_empty[n % PIECES]);
        if (warp != 0) continue;
        // Columns in pairs: int8 has 2 gq and 2 gq + 1 of each 16.  bf16 has gq and gq + 8:
        // lanes of even gq trade row 2 tq + 1 for row 2 tq of the lane after them.
#pragma unroll
        for (int nt = 0; nt < NR; ++nt) {
            float inv[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) inv[e] = !whole ? 1.f : lt[nt][e] == 0.f ? 0.f : 1.f / lt[nt][e];   // no key: zeros
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int row = nt * 8 + 2 * tq + e;
                if (!whole && gq == 0 && tile * ROWS + row < s.packed)
                    *reinterpret_cast<float2 *>(slot + ROWS * D + 2 * row) = make_float2(mt[nt][e], lt[nt][e]);
            }
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int u = 0; u < 2; ++u) {            // int8: a row; bf16: a column of gq
                    const int e = INT8 ? u : gq & 1;
                    float a, b;
                    if constexpr (INT8) {
                        a = o[nt][t][u] * inv[u];
                        b = o[nt][t][2 + u] * inv[u];
                    } else {
                        const float x0 = o[nt][t][2 * u] * inv[0], x1 = o[nt][t][2 * u + 1] * inv[1];
                        const float got = __shfl_xor_sync(0xffffffffu, e ? x0 : x1, 4);
                        a = e ? got : x0;
                        b = e ? x1 : got;
                    }
                    const int row = nt * 8 + 2 * tq + e, pr = tile * ROWS + row;
                    const int col = 16 * t + (INT8 ? 2 * gq : 8 * u + (gq & ~1));
                    if (pr >= s.packed) continue;
                    const int r = pr / group;
                    if (whole)
                        *reinterpret_cast<uint32_t *>(p.out + (int64_t)(s.row + r) * p.ldo +
                                                      (head * group + pr - r * group) * D + col) = pack_bf16(a, b);
                    else *reinterpret_cast<float2 *>(slot + row * D + col) = make_float2(a, b);
                }
            __syncwarp();
        }
    }
}

template <int FORM, int D, int NR, bool LONG = false>
echo_status launch(const echo::KvAttention &a, cudaStream_t st) {
    using C = Cfg<FORM, D, NR, LONG>;
    const bool p16 = FORM == kInt4 && a.pool->page_tokens == 16;
    auto *const kernel = p16 ? kv_decode_kernel<FORM, D, NR, LONG, FORM == kInt4> : kv_decode_kernel<FORM, D, NR, LONG, false>;
    static int attr_done[64][2] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && !attr_done[dev][p16]) {
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
        attr_done[dev][p16] = 1;
    }
    CUtensorMap tm, tm_scales = {};
    constexpr int most = FORM == kInt4 ? 32 : C::BK;
    const uint32_t tokens = (uint32_t)(a.pool->page_tokens < most ? a.pool->page_tokens : most);
    if (FORM == kInt4 ? !echo::make_tmap_code_pairs(&tm, *a.pool, tokens) || !echo::make_tmap_scale_pairs(&tm_scales, *a.pool, tokens)
                      : !echo::make_tmap_pages(&tm, *a.pool, tokens))
        return ECHO_ERR_CUDA;
    DecodeParams p;
    p.pool = echo::kv_pool(*a.pool);
    p.work = echo::kv_work(a, C::ROWS, C::ROWS, C::BSHIFT, 2 * echo::num_sms(), kWholeKeys);
    p.q = static_cast<const __nv_bfloat16 *>(a.q);
    p.out = static_cast<__nv_bfloat16 *>(a.out);
    p.ws = static_cast<float *>(a.ws);
    p.ldq = a.ldq;
    p.ldo = a.ldo;
    p.scale_log2 = 1.4426950408889634f / sqrtf((float)D) * (FORM == kInt4 ? kNibbleUnit : FORM == kInt8 ? kCodeUnit : 1.f);
    p.err = echo::device_error_ptr();
    cudaError_t launched;
    {
        echo::LaunchScope ls(ECHO_K_KV_ATTENTION, a.batch->n_rows, (int64_t)a.Hq * D, a.batch->n_seqs, st);
        launched = echo::launch_chained(kernel, dim3(p.work.workers), dim3(C::THREADS), C::SMEM, st, tm, tm_scales, p);
    }
    if (launched == cudaSuccess) echo::launch_kv_join(a, p.work, st);   // it needs what the kernel leaves
    return echo::last_launch_status();
}

// Packed rows of a tile for sequences of `rows`, 0: more than this kernel is for.  Measured
// with 8 sequences of 7800 tokens, 16 heads (us; the chunk kernel in brackets):
//   d 64:  bf16 8 rows 56, 16 56, 24 59, 32 64 (74), 48 in tiles of 24 84 (75)
//          int8 8 rows 35, 16 39, 24 47, 32 58 (100), 48 in 24s 75, 64 in 32s 92 (102)
//   d 128: bf16 8 rows 89, 16 90 (108), 24 in 16s 104, 32 103 (108, 110; one sequence of
//          32760 tokens, 40 heads: 32 in 16s 190, 133)
//          int8 8 rows 56, 16 60, 24 in 16s 89, 32 90 (128), 48 131 (129); three CTAs of an
//          SM, with two thirds of the registers, are slower: d 64 int8 24 rows 60
//   4 bits: d 64 9 rows 29, 24 32 (59), 32 42 (60), 48 in 24s 52 (60), 64 in 32s 69 (60);
//          d 128 16 41, 24 in 16s 67 (77), 32 68 (79), 48 (81)
int tile_rows(int form, int d, int64_t rows) {
    if (d == 128) return rows <= 8 ? 8 : rows <= (form != kBf16 ? 32 : 16) ? 16 : 0;
    if (rows <= 32) return (int)(rows + 7) / 8 * 8 + (rows == 0 ? 8 : 0);
    if (form != kBf16 && rows <= 48) return 24;
    return form == kInt8 && rows <= 64 ? 32 : 0;
}

template <int FORM, int D>
echo_status launch_rows(const echo::KvAttention &a, int tile, cudaStream_t st) {
    if constexpr (FORM == kInt4 && D == 64) {
        // 16 blocks of 256 keys for each worker, if the sequences are all as long as the longest may be
        const double keys = (double)echo::kv_longest(a);
        if (tile == 8 && (double)a.batch->n_seqs * a.pool->H * keys >= 2.0 * echo::num_sms() * 16 * 256)
            return launch<FORM, D, 1, true>(a, st);
    }
    if (tile == 8) return launch<FORM, D, 1>(a, st);
    if (tile == 16) return launch<FORM, D, 2>(a, st);
    if constexpr (D == 64) {
        if (tile == 24) return launch<FORM, D, 3>(a, st);
        return launch<FORM, D, 4>(a, st);
    }
    return ECHO_ERR_SHAPE;
}

}  // namespace

namespace echo {

size_t kv_decode_workspace(const echo_kv_pool &pool) {
    return kv_workspace_bytes(2 * num_sms(), kDecodeRows, pool.d);
}

bool kv_few_rows(const echo_kv_pool &pool, int64_t rows) {
    return tile_rows(pool.kind, pool.d, rows) > 0;
}

echo_status launch_kv_decode(const KvAttention &a, int64_t rows, cudaStream_t st) {
    const int form = a.pool->kind, tile = tile_rows(form, a.pool->d, rows);
    if (a.pool->d == 64)
        return form == kInt4 ? launch_rows<kInt4, 64>(a, tile, st)
               : form == kInt8 ? launch_rows<kInt8, 64>(a, tile, st) : launch_rows<kBf16, 64>(a, tile, st);
    return form == kInt4 ? launch_rows<kInt4, 128>(a, tile, st)
           : form == kInt8 ? launch_rows<kInt8, 128>(a, tile, st) : launch_rows<kBf16, 128>(a, tile, st);
}

}  // namespace echo
