// Attention of chunks of new rows over the paged cache, on the 5th-generation tensor
// cores.  An item is two tiles of up to 128 packed rows (row x head of a group) of one
// key/value head; one CTA per SM works through its share of all items (kv_schedule.cuh),
// 128 keys at a time, the two tiles in ping-pong so that one tile's softmax runs while the
// tensor cores work on the other:
//   warp 0      copies key blocks page by page (K_0, V_0, K_1, V_1, ...) into a ring of
//               shared-memory tiles (128-byte swizzle, 64-column boxes);
//   warp 1      one elected lane issues S_t = Q_t K^T (TMEM) and O_t += P_t V (P from
//               TMEM), in the order PV0_f S0_{f+1} PV1_f S1_{f+1}, across pieces too;
//   warp 2      tensor memory; bf16: clears the value rows that no row may use (below);
//   warp 3      walks the pieces, hands them to the other warps, copies the queries;
//   four warps  (int8) codes to bf16, a key per thread: the copy leaves a row of codes
//               where the second half of the row's bf16 values goes, so that each thread
//               overwrites only its own;
//   eight warps softmax of the two tiles, a row per thread: the running maximum comes from
//               the piece's first block and moves only when a block's weights sum to more
//               than 2^64 (exact after the division by the row sum).
// A row's weights are 0 where it does not see the key, but 0 times a value that is not
// finite is not 0: slots past a sequence's length may hold anything, and a later row's
// values too.  In the blocks that some row does not see whole, warp 2 therefore clears
// values past the end, clears those that are not finite and names their keys; a row that
// sees such a key becomes NaN.  For int8 pages only a scale can be non-finite: it then
// spoils the key's score, and stands as 0 among the values' scales.
// Every wait is bounded (ECHO_ERR_TIMEOUT).
#include <cfloat>

#include "kv_schedule.cuh"

namespace {

constexpr int BM = 128, TILES = 2, BN = 128;
constexpr int ATOM = 128 * 128;                 // 128 rows of 64 bf16
constexpr uint32_t TMEM_COLS = 512, O_COL = 256;
constexpr int PIECES = 4;                       // handed out ahead
constexpr int SLOT_ROWS = TILES * BM;
constexpr int V_AHEAD = 4;                      // value tiles in the ring are fewer

template <bool INT8, int D>
struct Cfg {
    static constexpr int THREADS = INT8 ? 512 : 384;
    static constexpr int SOFT0 = THREADS / 32 - 8;             // first softmax warp
    static constexpr int ATOMS = D / 64;
    static constexpr int Q_BYTES = ATOMS * ATOM;               // of a tile
    // int8 codes land at byte ATOM of their tile: for d 128 in its second half
    static constexpr int SLOT = INT8 && D == 64 ? ATOM + ATOM / 2 : ATOMS * ATOM;
    static constexpr int RING = D == 128 ? 5 : 6;
    static constexpr int TILES_BYTES = TILES * Q_BYTES + RING * SLOT;
    static constexpr uint32_t IDESC_S = idesc_bf16_f32(BM, BN);
    static constexpr uint32_t IDESC_PV = idesc_bf16_f32(BM, D) | (1u << 16);   // B MN-major
};

struct ChunkParams {
    KvPool pool;
    KvWork work;
    __nv_bfloat16 *out;
    float *ws;
    int64_t ldo;
    int tile_rows;           // packed rows of one of the two tiles
    float scale_log2;
    int *err;
};

struct Piece {
    int64_t shift;
    int blocks, kb0, keys, low;      // blocks < 0: no more pieces; low: keys that every row sees
    int row, packed, len, head, tile, seq;
    int whole, first;
};

// what shared memory holds beside the tiles
template <bool INT8, int D>
struct Side {
    static constexpr int RING = Cfg<INT8, D>::RING;
    uint64_t q_full, q_empty, full[RING], empty[RING], raw_full[RING], v_ok[V_AHEAD];
    uint64_t s_full[TILES], p_full[TILES], pv_done[TILES], drain;
    uint64_t piece_full[PIECES], piece_empty[PIECES], sc_full[2], sc_empty[2];
    Piece piece[PIECES];
    uint32_t spoilt[V_AHEAD][4];     // keys of a block with values that are not finite
    uint32_t tmem_slot;
    int abort_flag;
    union alignas(16) {              // read 16 bytes at a time
        KvFound found;
        float scales[INT8 ? 2 : 1][2][INT8 ? BN : 1];   // of blocks f & 1: keys, values
    };
};

template <bool INT8, int D>
__global__ void __launch_bounds__((Cfg<INT8, D>::THREADS), 1)
kv_chunk_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_kv,
                const ChunkParams p) {
    using C = Cfg<INT8, D>;
    constexpr int RING = C::RING;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t *Qs = smem, *Ring = smem + TILES * C::Q_BYTES;
    Side<INT8, D> &sh = *reinterpret_cast<Side<INT8, D> *>(smem + C::TILES_BYTES);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        // every barrier is waited for in each of its phases, in order, by whoever waits on
        // it, and none can be two phases ahead of a waiter
        mbar_init(&sh.q_full, 1);
        mbar_init(&sh.q_empty, 1);
        for (int i = 0; i < RING; ++i) {
            mbar_init(&sh.full[i], INT8 ? 4 : 1);
            mbar_init(&sh.empty[i], INT8 ? 1 : 2);     // the MMAs, and warp 2
            mbar_init(&sh.raw_full[i], 1);
        }
        for (int i = 0; i < V_AHEAD; ++i) mbar_init(&sh.v_ok[i], 1);
        for (int t = 0; t < TILES; ++t) {
            mbar_init(&sh.s_full[t], 1);
            mbar_init(&sh.p_full[t], 4);
            mbar_init(&sh.pv_done[t], 1);
        }
        mbar_init(&sh.drain, 1);
        for (int i = 0; i < PIECES; ++i) {
            mbar_init(&sh.piece_full[i], 1);
            mbar_init(&sh.piece_empty[i], INT8 ? 2 + 4 + 8 : 3 + 8);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.sc_full[i], 4);
            mbar_init(&sh.sc_empty[i], 8);
        }
        sh.abort_flag = 0;
        fence_barrier_init();
        tma_prefetch_desc(&tm_q);
        tma_prefetch_desc(&tm_kv);
    }
    if (warp == 2) tmem_alloc(&sh.tmem_slot, TMEM_COLS);
    // query rows that no copy reaches (groups that do not divide 128) are zeros
    for (int i = threadIdx.x; i < (BM - p.tile_rows) * TILES * C::ATOMS * 8; i += C::THREADS) {
        const int r = p.tile_rows + (i >> 3) % (BM - p.tile_rows), a = (i >> 3) / (BM - p.tile_rows);
        *reinterpret_cast<uint4 *>(Qs + a * ATOM + r * 128 + (i & 7) * 16) = make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem_slot;
    volatile int *abort_v = &sh.abort_flag;
    pdl_enter();
    KvWalk walk;
    kv_find<C::THREADS, false>(p.work, blockIdx.x, sh.found, walk);
    __syncthreads();                     // `found` makes room for the scales
    auto wait_all = [&](uint64_t *bar, uint32_t parity) -> bool {
        return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_v, p.err));
    };
    // the n-th piece, once it is there
    auto piece = [&](int n, bool &ok) -> const Piece & {
        ok = wait_all(&sh.piece_full[n % PIECES], (n / PIECES) & 1);
        return sh.piece[n % PIECES];
    };
    auto piece_done = [&](int n) {
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.piece_empty[n % PIECES]);
    };

    if (warp < 4) {
        if constexpr (INT8) asm volatile("setmaxnreg.dec.sync.aligned.u32 48;" ::: "memory");
        else asm volatile("setmaxnreg.dec.sync.aligned.u32 48;" ::: "memory");
        bool ok = true;
        if (warp == 3) {
            // ---------------- pieces, and their queries ----------------
            int n = 0, loads = 0;
            for (bool more = true; more; ++n) {
                more = walk.next(p.work);
                if (n >= PIECES && !wait_all(&sh.piece_empty[n % PIECES], ((n / PIECES) & 1) ^ 1)) break;
                Piece &pc = sh.piece[n % PIECES];
                if (lane == 0) {
                    pc.blocks = more ? walk.kb1 - walk.kb0 : -1;
                    if (more) {
                        pc.shift = walk.s.shift;
                        pc.kb0 = walk.kb0;
                        pc.keys = walk.s.keys(p.work, walk.tile);
                        pc.low = min(pc.keys, walk.s.top(p.work, walk.s.row + walk.tile * p.work.tile / p.work.group));
                        pc.row = walk.s.row;
                        pc.packed = walk.s.packed;
                        pc.len = walk.s.len;
                        pc.head = walk.head;
                        pc.tile = walk.tile;
                        pc.seq = walk.seq;
                        pc.whole = walk.whole();
                        pc.first = walk.first;
                        if (walk.s.len > p.work.cap) echo_flag_error(p.err, ECHO_ERR_PAGE);
                    }
                    mbar_arrive(&sh.piece_full[n % PIECES]);
                }
                __syncwarp();
                if (!more || walk.kb0 == walk.kb1) continue;
                // the queries' buffer is free once the last S of the piece before is done
                if (loads > 0 && !wait_all(&sh.q_empty, (loads - 1) & 1)) break;
                if (lane == 0) {
                    mbar_arrive_expect_tx(&sh.q_full, TILES * C::ATOMS * p.tile_rows * 128);
                    const int tokens = p.tile_rows / p.work.group;
                    for (int t = 0; t < TILES; ++t)
                        for (int a = 0; a < C::ATOMS; ++a)
                            tma_load_3d(Qs + t * C::Q_BYTES + a * ATOM, &tm_q, &sh.q_full, 64 * a,
                                        walk.head * p.work.group,
                                        walk.s.row + (walk.tile * TILES + t) * tokens);
                }
                ++loads;
            }
            if (*abort_v && loads > 0)
                mbar_wait(&sh.q_full, (loads - 1) & 1, abort_v, nullptr, 100000000ull);
        } else if (warp == 0) {
            // ---------------- keys and values, a page at a time ----------------
            const int shift = p.pool.shift, per_block = BN >> shift;
            int li = 0;                                       // copies into the ring so far
            for (int n = 0; ok; ++n) {
                const Piece &pc = piece(n, ok);
                if (!ok || pc.blocks < 0) break;
                const int kb0 = pc.kb0, kb1 = kb0 + pc.blocks, head = pc.head, keys = pc.keys;
                const int32_t *table = p.work.b.table + (int64_t)pc.seq * p.work.b.max_pages;
                piece_done(n);
                const int pages = (keys + (1 << shift) - 1) >> shift;
                auto page_of = [&](int i) -> int {
                    if (i >= pages) return 0;
                    const int page = table[i];
                    if ((unsigned)page < (unsigned)p.pool.n_pages) return page;
                    echo_flag_error(p.err, ECHO_ERR_PAGE);
                    return 0;
                };
                if (kb0 == kb1) continue;
                // 32 pages in the lanes, the next 32 on their way
                int c0 = kb0 * per_block;
                int now = page_of(c0 + lane), then = page_of(c0 + 32 + lane);
                for (int kb = kb0; kb < kb1; ++kb) {
                    const int first = kb * per_block;
                    if (first >= c0 + 32) {
                        c0 += 32;
                        now = then;
                        then = page_of(c0 + 32 + lane);
                    }
                    const int some = min(per_block, pages - first);
                    const int page = __shfl_sync(0xffffffffu, now, (first - c0 + lane) & 31);
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv, ++li) {
                        const int slot = li % RING;
                        ok = wait_all(&sh.empty[slot], ((li / RING) & 1) ^ 1);
                        if (!ok) break;
                        uint64_t *bar = INT8 ? &sh.raw_full[slot] : &sh.full[slot];
                        uint8_t *dst = Ring + slot * C::SLOT;
                        // int8: both scales come with the keys
                        if (lane == 0)
                            mbar_arrive_expect_tx(bar, (uint32_t)(some << shift) * (INT8 ? D + (kv ? 0 : 8) : 2 * D));
                        __syncwarp();
                        if (lane < some) {
                            const int z = (page * 2 + kv) * p.pool.H + head, r0 = lane << shift;
                            if constexpr (INT8) {
                                tma_load_3d(dst + ATOM + r0 * D, &tm_kv, bar, 0, 0, z);
                                if (kv == 0) {
                                    // the scales of 32 keys where their own warp's rows will be:
                                    // it reads them before it writes
                                    const int step = min(shift, 5);
                                    for (int r = 0; r < 1 << shift; r += 1 << step) {
                                        uint8_t *at = dst + ((r0 + r) & ~31) * 128 + ((r0 + r) & 31) * 4;
                                        const float *src = p.pool.scale + (((int64_t)z << shift) + r);
                                        bulk_load_1d(at, src, 4u << step, bar);
                                        bulk_load_1d(at + 128, src + ((int64_t)p.pool.H << shift), 4u << step, bar);
                                    }
                                }
                            } else {
#pragma unroll
                                for (int a = 0; a < C::ATOMS; ++a)
                                    tma_load_3d(dst + a * ATOM + r0 * 128, &tm_kv, bar, 64 * a, 0, z);
                            }
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                }
            }
            if (*abort_v && lane == 0)   // let this CTA's copies land before it exits
                for (int i = max(0, li - RING); i < li; ++i)
                    mbar_wait(INT8 ? &sh.raw_full[i % RING] : &sh.full[i % RING], (i / RING) & 1, abort_v,
                              nullptr, 100000000ull);
        } else if (warp == 1) {
            // ---------------- MMA issuer (see attn_tc_kernel of attention.cu) ----------------
            const bool leader = elect_one_sync();
            constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
            constexpr uint32_t LO_K = 1u << 16;
            constexpr uint32_t LO_MN = (uint32_t)(ATOM >> 4) << 16;
            const uint32_t q_lo = ((smem_u32(Qs) & 0x3FFFFu) >> 4) | LO_K;
            const uint32_t ring_lo = (smem_u32(Ring) & 0x3FFFFu) >> 4;
            auto desc = [](uint32_t lo) -> uint64_t { return ((uint64_t)DESC_HI << 32) | lo; };
            auto mma_s = [&](int t, int slot) {
                const uint32_t a_lo = q_lo + (uint32_t)t * (C::Q_BYTES >> 4);
                const uint32_t b_lo = (ring_lo + (uint32_t)slot * (C::SLOT >> 4)) | LO_K;
                const uint32_t d = tmem + (uint32_t)(t * BN);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    const uint32_t off = (uint32_t)(((kk >> 2) * ATOM + (kk & 3) * 32) >> 4);
                    tc_mma_f16(d, desc(a_lo + off), desc(b_lo + off), C::IDESC_S, kk > 0);
                }
            };
            auto mma_pv = [&](int t, int slot, uint32_t acc0) {
                const uint32_t b_lo = (ring_lo + (uint32_t)slot * (C::SLOT >> 4)) | LO_MN;
                const uint32_t d = tmem + O_COL + (uint32_t)(t * D);
                const uint32_t a = tmem + (uint32_t)(t * BN);
                tc_mma_f16_tmem_a(d, a, desc(b_lo), C::IDESC_PV, acc0);
#pragma unroll
                for (int kk = 1; kk < BN / 16; ++kk)
                    tc_mma_f16_tmem_a(d, a + 8 * kk, desc(b_lo + (uint32_t)(kk * 2048 >> 4)), C::IDESC_PV, 1u);
            };
            // the blocks of the next piece that has any, 0 at the end
            int n = 0, pieces = 0;                            // taken, and those with blocks
            auto next_blocks = [&]() -> int {
                for (;;) {
                    const Piece &pc = piece(n, ok);
                    if (!ok || pc.blocks < 0) return 0;
                    const int b = pc.blocks;
                    piece_done(n);
                    ++n;
                    if (b > 0) return b;
                }
            };
            int slot = 0;                                     // of K_f; V_f and K_{f+1} follow
            uint32_t ph = 0;
            auto next = [&](int &s, uint32_t &h) { if (++s == RING) { s = 0; h ^= 1u; } };
            int left = next_blocks();                         // of the piece, block f included
            if (left > 0 && ok) {
                ok = wait_all(&sh.q_full, 0) && wait_all(&sh.full[0], 0);
                if (ok) {
                    tc_fence_after();
                    if (leader) {
                        mma_s(0, 0);
                        tc_commit(&sh.s_full[0]);
                        mma_s(1, 0);
                        tc_commit(&sh.s_full[1]);
                        tc_commit(&sh.empty[0]);
                        if (left == 1) tc_commit(&sh.q_empty);
                    }
                    __syncwarp();
                }
            }
            uint32_t acc = 0;
            for (int f = 0; ok && left > 0; ++f) {
                int vs = slot; uint32_t vph = ph; next(vs, vph);
                int ks = vs; uint32_t kph = vph; next(ks, kph);
                const bool last = left == 1;
                // after the last block the next piece's: known before this block's P V
                const int then = last ? next_blocks() : left - 1;
                if (!ok) break;
                if (!wait_all(&sh.p_full[0], f & 1)) { ok = false; break; }
                if (!(INT8 ? wait_all(&sh.full[vs], vph) : wait_all(&sh.v_ok[f % V_AHEAD], (f / V_AHEAD) & 1))) { ok = false; break; }
                tc_fence_after();
                if (leader) {
                    mma_pv(0, vs, acc);
                    if (last) tc_commit(&sh.pv_done[0]);
                }
                __syncwarp();
                if (then > 0) {
                    if (last && !wait_all(&sh.q_full, ++pieces & 1)) { ok = false; break; }
                    if (!wait_all(&sh.full[ks], kph)) { ok = false; break; }
                    tc_fence_after();
                    if (leader) {
                        mma_s(0, ks);
                        tc_commit(&sh.s_full[0]);
                    }
                    __syncwarp();
                }
                if (!wait_all(&sh.p_full[1], f & 1)) { ok = false; break; }
                tc_fence_after();
                if (leader) {
                    mma_pv(1, vs, acc);
                    tc_commit(&sh.empty[vs]);
                    if (last) tc_commit(&sh.pv_done[1]);
                    if (then > 0) {
                        mma_s(1, ks);
                        tc_commit(&sh.s_full[1]);
                        tc_commit(&sh.empty[ks]);
                        if (then == 1) tc_commit(&sh.q_empty);
                    }
                }
                __syncwarp();
                acc = last ? 0u : 1u;
                left = then;
                slot = ks;
                ph = kph;
            }
            if (!ok && leader) {   // the MMAs already issued, before tensor memory is freed
                tc_commit(&sh.drain);
                mbar_wait(&sh.drain, 0, abort_v, nullptr, 100000000ull);
            }
            __syncwarp();
        } else if (!INT8) {
            // ---------------- values that no row may use, cleared ----------------
            int f = 0;
            for (int n = 0; ok; ++n) {
                const Piece &pc = piece(n, ok);
                if (!ok || pc.blocks < 0) break;
                const int kb0 = pc.kb0, kb1 = kb0 + pc.blocks, keys = pc.keys, low = pc.low;
                piece_done(n);
                for (int kb = kb0; kb < kb1; ++kb, ++f) {
                    // every copy is seen here before its tile is filled again
                    ok = wait_all(&sh.full[2 * f % RING], (2 * f / RING) & 1);
                    if (!ok) break;
                    if (lane == 0) mbar_arrive(&sh.empty[2 * f % RING]);
                    const int li = 2 * f + 1, slot = li % RING;
                    ok = wait_all(&sh.full[slot], (li / RING) & 1);
                    if (!ok) break;
                    if ((kb + 1) * BN > low) {
                        const int valid = keys - kb * BN;
                        uint32_t spoilt[4] = {0, 0, 0, 0};
                        // a lane's chunk of a row, four rows (or eight) at a time
#pragma unroll 4
                        for (int i = lane; i < BN * C::ATOMS * 8; i += 32) {
                            const int r = (i >> 3) % BN, a = (i >> 3) / BN;
                            uint4 *at = reinterpret_cast<uint4 *>(Ring + slot * C::SLOT + a * ATOM + r * 128) + (i & 7);
                            const uint4 v = *at;
                            // a bf16 is not finite if all bits of its exponent are set
                            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
                            bool bad = false;
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                bad |= (w[e] & 0x7F80u) == 0x7F80u || (w[e] & 0x7F800000u) == 0x7F800000u;
                            if (r >= valid || bad) {
                                *at = make_uint4(0, 0, 0, 0);
                                if (r < valid) spoilt[r >> 5] |= 1u << (r & 31);
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t all = __reduce_or_sync(0xffffffffu, spoilt[e]);
                            if (lane == 0) sh.spoilt[f % V_AHEAD][e] = all;
                        }
                        fence_proxy_async_smem();
                    }
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(&sh.v_ok[f % V_AHEAD]);
                        mbar_arrive(&sh.empty[slot]);
                    }
                }
            }
        }
    } else if (INT8 && warp < 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 48;" ::: "memory");
        // ---------------- codes to bf16, a key per thread ----------------
        const int r = (int)threadIdx.x - 128;                 // key of the block
        bool ok = true;
        int f = 0;
        for (int n = 0; ok; ++n) {
            const Piece &pc = piece(n, ok);
            if (!ok || pc.blocks < 0) break;
            const int kb0 = pc.kb0, kb1 = kb0 + pc.blocks, keys = pc.keys;
            piece_done(n);
            for (int kb = kb0; ok && kb < kb1; ++kb, ++f) {
#pragma unroll 1
                for (int kv = 0; kv < 2; ++kv) {
                    const int li = 2 * f + kv, slot = li % RING;
                    ok = wait_all(&sh.raw_full[slot], (li / RING) & 1);
                    if (!ok) break;
                    uint8_t *tile = Ring + slot * C::SLOT;
                    if (kv == 0) {
                        const float *sc = reinterpret_cast<const float *>(tile + (r & ~31) * 128) + lane;
                        float ks = sc[0], vs = sc[32];
                        __syncwarp();                         // read before the rows are written
                        const bool there = kb * BN + r < keys;
                        if (!(fabsf(vs) < INFINITY)) ks = NAN, vs = 0.f;
                        if (!there) ks = vs = 0.f;            // slots past the end: anything
                        ok = wait_all(&sh.sc_empty[f & 1], ((f >> 1) & 1) ^ 1);
                        if (!ok) break;
                        sh.scales[f & 1][0][r % (INT8 ? BN : 1)] = ks * p.scale_log2;
                        sh.scales[f & 1][1][r % (INT8 ? BN : 1)] = vs;
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&sh.sc_full[f & 1]);
                    }
#pragma unroll
                    for (int a = 0; a < C::ATOMS; ++a) {
                        uint4 in[4];                          // 64 codes of the row
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const int at = D == 128 ? r * 128 + (((4 * a + c) ^ (r & 7)) << 4)
                                                    : r * 64 + ((c ^ ((r >> 1) & 3)) << 4);
                            in[c] = *reinterpret_cast<const uint4 *>(tile + ATOM + at);
                        }
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const uint32_t w[4] = {in[c].x, in[c].y, in[c].z, in[c].w};
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const uint4 v = make_uint4(kv_codes2(w[2 * h], 0x4140), kv_codes2(w[2 * h], 0x4342),
                                                           kv_codes2(w[2 * h + 1], 0x4140), kv_codes2(w[2 * h + 1], 0x4342));
                                const int out = 2 * c + h;    // 8 values
                                *reinterpret_cast<uint4 *>(tile + a * ATOM + r * 128 + ((out ^ (r & 7)) << 4)) = v;
                            }
                        }
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.full[slot]);
                }
            }
        }
    } else {
        if constexpr (INT8) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;" ::: "memory");
        else asm volatile("setmaxnreg.inc.sync.aligned.u32 224;" ::: "memory");
        // ---------------- softmax and output of tile t, a row per thread ----------------
        const int t = (warp - C::SOFT0) >> 2, quad = warp & 3;
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        const uint32_t s_at = tmem + lane_base + (uint32_t)(t * BN);
        const uint32_t o_at = tmem + lane_base + O_COL + (uint32_t)(t * D);
        const int row = quad * 32 + lane;                     // of the tile
        bool ok = true;
        int f = 0, with_blocks = 0;
        for (int n = 0; ok; ++n) {
            const Piece &pc = piece(n, ok);
            if (!ok || pc.blocks < 0) break;
            const int pr = (pc.tile * TILES + t) * p.tile_rows + row;        // packed row
            const bool real = row < p.tile_rows && pr < pc.packed;
            int lim = pc.keys;                                // keys that the row sees
            if (real) {
                KvSeq s;
                s.len = pc.len;
                s.shift = pc.shift;
                lim = s.top(p.work, pc.row + pr / p.work.group);
            }
            const int warp_low = __reduce_min_sync(0xffffffffu, lim);
            const int kb0 = pc.kb0, blocks = pc.blocks, low = pc.low;
            float m = -FLT_MAX, l = 0.f;
            for (int j = 0; j < blocks; ++j, ++f) {
                ok = wait_all(&sh.s_full[t], f & 1);
                if (!ok) break;
                tc_fence_after();
                const int key0 = (kb0 + j) * BN;
                float sv[BN];
                const float sl2 = INT8 ? 1.f : p.scale_log2;
                const float *vsc = sh.scales[f & (INT8 ? 1 : 0)][1];
                if constexpr (INT8) {
                    ok = wait_all(&sh.sc_full[f & 1], (f >> 1) & 1);
                    if (!ok) break;
                }
                // the row's scores; -inf where it does not see the key
                auto load_s = [&]() {
#pragma unroll
                    for (int c = 0; c < BN / 32; ++c)
                        tmem_ld32(s_at + 32 * c, reinterpret_cast<uint32_t *>(sv + 32 * c));
                    tmem_ld_wait();
                    if constexpr (INT8) {
                        const float4 *ksc = reinterpret_cast<const float4 *>(sh.scales[f & 1][0]);
#pragma unroll
                        for (int i = 0; i < BN / 4; ++i) {
                            const float4 k4 = ksc[i];
                            f2_unpack(f2_mul(f2_pack(sv[4 * i], sv[4 * i + 1]), f2_pack(k4.x, k4.y)),
                                      sv[4 * i], sv[4 * i + 1]);
                            f2_unpack(f2_mul(f2_pack(sv[4 * i + 2], sv[4 * i + 3]), f2_pack(k4.z, k4.w)),
                                      sv[4 * i + 2], sv[4 * i + 3]);
                        }
                    }
                    if (key0 + BN > warp_low) {
                        const int seen = lim - key0;
#pragma unroll
                        for (int i = 0; i < BN; ++i)
                            if (i >= seen) sv[i] = -INFINITY;
                    }
                };
                load_s();
                auto block_max = [&]() -> float {
                    float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int i = 0; i < BN; i += 8) {
                        m4[0] = fmax3(m4[0], sv[i], sv[i + 1]);
                        m4[1] = fmax3(m4[1], sv[i + 2], sv[i + 3]);
                        m4[2] = fmax3(m4[2], sv[i + 4], sv[i + 5]);
                        m4[3] = fmax3(m4[3], sv[i + 6], sv[i + 7]);
                    }
                    return fmaxf(fmax3(m4[0], m4[1], m4[2]), m4[3]);
                };
                // P = 2^(s - m) on fp32 pairs, times the values' scales, in bf16 pairs;
                // returns the row's sum of 2^(s - m)
                uint32_t pk[BN / 2];
                auto exp_pass = [&]() -> float {
                    const uint64_t scale2 = f2_pack(sl2, sl2), negm2 = f2_pack(-m, -m);
                    uint64_t acc2[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
                    for (int i = 0; i < BN / 2; ++i) {
                        float x0, x1;
                        if constexpr (INT8) f2_unpack(f2_add(f2_pack(sv[2 * i], sv[2 * i + 1]), negm2), x0, x1);
                        else f2_unpack(f2_fma(f2_pack(sv[2 * i], sv[2 * i + 1]), scale2, negm2), x0, x1);
                        float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
                        acc2[i & 3] = f2_add(acc2[i & 3], f2_pack(p0, p1));
                        if constexpr (INT8) {
                            const float2 v2 = reinterpret_cast<const float2 *>(vsc)[i];
                            f2_unpack(f2_mul(f2_pack(p0, p1), f2_pack(v2.x, v2.y)), p0, p1);
                        }
                        pk[i] = pack_bf16(p0, p1);
                    }
                    float a0, a1;
                    f2_unpack(f2_add(f2_add(acc2[0], acc2[1]), f2_add(acc2[2], acc2[3])), a0, a1);
                    return a0 + a1;
                };
                // a first block that shows the row no key leaves the maximum at the lowest
                // number: P is 0 there, and the first finite score overflows and brings its own
                if (j == 0) m = fmaxf(block_max() * sl2, -FLT_MAX);
                float bsum = exp_pass();
                const bool redo = !(bsum <= 1.8446744e19f);     // > 2^64, inf or NaN
                if (__any_sync(0xffffffffu, redo)) {
                    load_s();                                   // its registers hold P
                    float alpha = 1.f;
                    if (redo) {
                        const float m_new = fmaxf(m, block_max() * sl2);
                        alpha = ex2_approx(m - m_new);
                        l *= alpha;
                        m = m_new;
                    }
                    if (j > 0) {   // S of this block completed after P V of the one before
#pragma unroll
                        for (int c = 0; c < D / 32; ++c) {
                            uint32_t o[32];
                            tmem_ld32(o_at + 32 * c, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                            tmem_st32(o_at + 32 * c, o);
                        }
                        tmem_st_wait();
                    }
                    bsum = exp_pass();
                }
                l += bsum;
                tmem_st32(s_at, pk);
                tmem_st32(s_at + 32, pk + 32);
                tmem_st_wait();
                if (!INT8 && key0 + BN > low) {                 // keys whose values are not finite
                    ok = wait_all(&sh.v_ok[f % V_AHEAD], (f / V_AHEAD) & 1);
                    if (!ok) break;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int seen = lim - key0 - 32 * e;
                        const uint32_t mask = seen >= 32 ? 0xffffffffu : seen > 0 ? (1u << seen) - 1u : 0u;
                        if (sh.spoilt[f % V_AHEAD][e] & mask) l = NAN;
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&sh.p_full[t]);
                    if constexpr (INT8) mbar_arrive(&sh.sc_empty[f & 1]);
                }
            }
            if (!ok) break;
            if (blocks > 0) {
                ok = wait_all(&sh.pv_done[t], with_blocks++ & 1);
                if (!ok) break;
                tc_fence_after();
            }
            const bool whole = pc.whole;
            const float inv = l == 0.f ? 0.f : 1.f / l;          // no key: zeros
            __nv_bfloat16 *dst = nullptr;
            float *part = nullptr;
            if (real) {
                const int g = p.work.group;
                dst = p.out + (int64_t)(pc.row + pr / g) * p.ldo + (pc.head * g + pr % g) * D;
            }
            const int slot_row = t * p.tile_rows + row;
            if (!whole) {
                part = kv_slot(p.ws, blockIdx.x, pc.first, SLOT_ROWS, D);
                if (real) *reinterpret_cast<float2 *>(part + SLOT_ROWS * D + 2 * slot_row) = make_float2(m, l);
                part += (int64_t)slot_row * D;
            }
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                uint32_t o[32];
                if (blocks > 0) {
                    tmem_ld32(o_at + 32 * c, o);
                    tmem_ld_wait();
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = 0u;
                }
                if (real && whole) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float v[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(o[8 * i + e]) * inv;
                        *reinterpret_cast<uint4 *>(dst + 32 * c + 8 * i) = pack8_bf16(v);
                    }
                } else if (real) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        *reinterpret_cast<uint4 *>(part + 32 * c + 4 * i) =
                            make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
                }
                __syncwarp();            // tensor memory is read by whole warps
            }
            tc_fence_before();           // O is out of tensor memory before the next P is announced
            piece_done(n);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 2) {
        tc_fence_after();
        tmem_dealloc(tmem, TMEM_COLS);
    }
}

template <bool INT8, int D>
echo_status launch(const echo::KvAttention &a, cudaStream_t st) {
    using C = Cfg<INT8, D>;
    constexpr int SMEM = C::TILES_BYTES + (int)sizeof(Side<INT8, D>);
    using S = Side<INT8, D>;
    static_assert(SMEM <= 232448 && C::TILES_BYTES % 16 == 0 && offsetof(S, scales) % 16 == 0, "");
    static int attr_done[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && !attr_done[dev]) {
        cudaFuncSetAttribute(kv_chunk_kernel<INT8, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
        attr_done[dev] = 1;
    }
    const int group = a.Hq / a.pool->H, tokens = BM / group;
    CUtensorMap tq, tk;
    if (!echo::make_tmap_rows(&tq, a.q, (uint64_t)a.batch->n_rows, (uint64_t)a.Hq, (uint64_t)D, (uint64_t)a.ldq,
                              (uint32_t)group, (uint32_t)tokens) ||
        !echo::make_tmap_pages(&tk, *a.pool, (uint32_t)a.pool->page_tokens))
        return ECHO_ERR_CUDA;
    ChunkParams p;
    p.pool = echo::kv_pool(*a.pool);
    p.tile_rows = tokens * group;
    p.work = echo::kv_work(a, TILES * p.tile_rows, SLOT_ROWS, 7, echo::num_sms());
    p.out = static_cast<__nv_bfloat16 *>(a.out);
    p.ws = static_cast<float *>(a.ws);
    p.ldo = a.ldo;
    p.scale_log2 = 1.4426950408889634f / sqrtf((float)D);
    p.err = echo::device_error_ptr();
    {
        echo::LaunchScope ls(ECHO_K_KV_ATTENTION, a.batch->n_rows, (int64_t)a.Hq * D, a.batch->n_seqs, st);
        echo::launch_chained(kv_chunk_kernel<INT8, D>, dim3(p.work.workers), dim3(C::THREADS), SMEM, st, tq, tk, p);
    }
    echo::launch_kv_join(a, p.work, st);
    return echo::last_launch_status();
}

}  // namespace

namespace echo {

size_t kv_chunk_workspace(const echo_kv_pool &pool) {
    return kv_workspace_bytes(num_sms(), SLOT_ROWS, pool.d);
}

echo_status launch_kv_chunk(const KvAttention &a, cudaStream_t st) {
    const bool i8 = a.pool->kind == ECHO_CACHE_INT8;
    if (a.pool->d == 64) return i8 ? launch<true, 64>(a, st) : launch<false, 64>(a, st);
    return i8 ? launch<true, 128>(a, st) : launch<false, 128>(a, st);
}

}  // namespace echo
