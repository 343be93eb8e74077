// Attention of chunks of new rows over the paged cache, on the 5th-generation tensor
// cores.  An item is two tiles of up to 128 packed rows (row x head of a group) of one
// key/value head; one CTA per SM works through its share of all items (kv_schedule.cuh),
// 128 keys at a time, the two tiles in ping-pong so that one tile's softmax runs while the
// tensor cores work on the other:
//   warp 0      copies key blocks page by page (K_0, V_0, K_1, V_1, ...) into a ring of
//               shared-memory tiles (128-byte swizzle, 64-column boxes);
//   warp 1      one elected lane issues S_t = Q_t K^T (TMEM) and O_t += P_t V (P from
//               TMEM), in the order PV0_f S0_{f+1} PV1_f S1_{f+1}, across pieces too; for
//               heads of 64 S is half a block further ahead;
//   warp 3      walks the pieces, hands them to the other warps, copies the queries;
//   four warps  int8: codes to bf16, a key per thread: the copy leaves a row of codes where
//               the second half of the row's bf16 values goes, so that each thread
//               overwrites only its own.  bf16: clear values that no row may use (below);
//   eight warps softmax of the two tiles: a row's running maximum comes from
//               the piece's first block and moves only when a block's weights sum to more
//               than 2^64 (exact after the division by the row sum).
// A row's weights are 0 where it does not see the key, but 0 times a value that is not
// finite is not 0: slots past a sequence's length may hold anything, and a later row's
// values too.  In the blocks that some row does not see whole, four warps therefore clear
// values past the end, clear those that are not finite and name their keys; a row that
// sees such a key becomes NaN.  For int8 pages only a scale can be non-finite: it then
// spoils the key's score, and stands as 0 among the values' scales.
// Every wait is bounded (ECHO_ERR_TIMEOUT).
#include <cfloat>
#include <type_traits>

#include "kv_schedule.cuh"

namespace {

constexpr int BM = 128, TILES = 2, BN = 128;
constexpr int ATOM = 128 * 128;                 // 128 rows of 64 bf16
constexpr uint32_t TMEM_COLS = 512;
constexpr int PIECES = 4;                       // handed out ahead
constexpr int SLOT_ROWS = TILES * BM;
constexpr int kWholeKeys = 1024;                // 64 bf16 rows, 8 heads of 128: whole 512 keys 16.5 us, 1024 21.5; divided 19.8, 21.8
constexpr int PAIRS = 3;                        // (V_f, K_{f+1}) on their way or in use
constexpr int SPOILT = 2;                       // blocks whose spoilt keys are kept

template <bool INT8, int D>
struct Cfg {
    // warps 0-3, helpers from 4 on, softmax
    static constexpr int HELP = 4, SOFT0 = 4 + HELP, THREADS = 32 * (SOFT0 + 8);
    static constexpr int ATOMS = D / 64;
    static constexpr int Q_BYTES = ATOMS * ATOM;               // of a tile
    // int8 codes land at byte ATOM of their tile: for d 128 in its second half
    static constexpr int SLOT = INT8 && D == 64 ? ATOM + ATOM / 2 : ATOMS * ATOM;
    static constexpr int RING = D == 128 ? 5 : 6;              // d 64: of three blocks, below
    // tensor memory: S buffers of 128 columns, then O of both tiles.  d 64 leaves room for a
    // third S, and for the queries of two pieces (below, at the products)
    static constexpr int S_BUFS = D == 64 ? 3 : 2, Q_BUFS = D == 64 ? 2 : 1;
    static constexpr int S_BARS = D == 64 ? 6 : 2;   // full: one per buffer and tile that uses it
    static constexpr uint32_t O_COL = S_BUFS * BN;
    static constexpr int Q_BUF = TILES * Q_BYTES, TILES_BYTES = Q_BUFS * Q_BUF + RING * SLOT;
    // registers of warps 0-3, of four helpers and of four softmax warps: together at most
    // what the launch gives; the splits that were fastest.  4864 rows, 8 heads, bf16: 32768
    // keys of 128 354 us (72, 24, 208: 358), 8192 keys of 64 70 us (96, 48, 184: 73); int8
    // 464 and 98 us (88, 40, 192: 524 and 114; 56, 56, 200: 472 and 101), since then 472 and 97
    static constexpr int REGS[3] = {INT8 ? 64 : 88, INT8 ? 64 : 40, 192};
    static_assert(REGS[0] + HELP / 4 * REGS[1] + 2 * REGS[2] <= THREADS / 128 * (65536 / THREADS / 8 * 8),
                  "setmaxnreg takes from the launch's registers");
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

// the first blocks of a piece that every row sees whole
ECHO_DEV int kv_clear(const KvPiece &pc) { return min(max(pc.low / BN - pc.kb0, 0), max(pc.blocks, 0)); }

// what shared memory holds beside the tiles
template <bool INT8, int D>
struct Side {
    static constexpr int RING = Cfg<INT8, D>::RING;
    using C = Cfg<INT8, D>;
    uint64_t q_full[C::Q_BUFS], q_empty[C::Q_BUFS], k_first, pair[PAIRS], empty[RING], raw_full[RING], edge_go, v_ok;
    uint64_t s_full[C::S_BARS], p_full[C::S_BUFS], pv_done[TILES], drain;
    uint64_t piece_full[PIECES], piece_empty[PIECES], sc_full[2], sc_empty[2];
    KvPiece piece[PIECES];
    uint32_t spoilt[SPOILT][4];      // keys of a block with values that are not finite
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
    uint8_t *Qs = smem, *Ring = smem + C::Q_BUFS * C::Q_BUF;
    Side<INT8, D> &sh = *reinterpret_cast<Side<INT8, D> *>(smem + C::TILES_BYTES);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        // every barrier is waited for in each of its phases, in order, by whoever waits on
        // it, and none can be two phases ahead of a waiter
        for (int i = 0; i < C::Q_BUFS; ++i) {
            mbar_init(&sh.q_full[i], 1);
            mbar_init(&sh.q_empty[i], 1);
        }
        // V_f and K_{f+1} share a barrier: two copies, or two tiles from four warps
        mbar_init(&sh.k_first, INT8 ? 4 : 1);
        for (int i = 0; i < PAIRS; ++i) mbar_init(&sh.pair[i], INT8 ? 8 : 2);
        for (int i = 0; i < RING; ++i) {
            mbar_init(&sh.empty[i], 1);
            mbar_init(&sh.raw_full[i], 1);
        }
        mbar_init(&sh.edge_go, 1);
        mbar_init(&sh.v_ok, 4);
        for (int t = 0; t < TILES; ++t) {
            mbar_init(&sh.pv_done[t], 1);
        }
        for (int i = 0; i < C::S_BARS; ++i) mbar_init(&sh.s_full[i], 1);
        for (int i = 0; i < C::S_BUFS; ++i) mbar_init(&sh.p_full[i], 4);
        mbar_init(&sh.drain, 1);
        for (int i = 0; i < PIECES; ++i) {
            mbar_init(&sh.piece_full[i], 1);
            mbar_init(&sh.piece_empty[i], 2 + C::HELP + 8);
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
    for (int i = threadIdx.x; i < (BM - p.tile_rows) * C::Q_BUFS * TILES * C::ATOMS * 8; i += C::THREADS) {
        const int r = p.tile_rows + (i >> 3) % (BM - p.tile_rows), a = (i >> 3) / (BM - p.tile_rows);
        *reinterpret_cast<uint4 *>(Qs + a * ATOM + r * 128 + (i & 7) * 16) = make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // through a warp-wide reduction, whose result the compiler knows to be the same in every
    // lane: addresses and descriptors made from it need no transfer to uniform registers
    const uint32_t tmem = __reduce_max_sync(0xffffffffu, sh.tmem_slot);
    volatile int *abort_v = &sh.abort_flag;
    pdl_enter();
    KvWalk walk;
    kv_find<C::THREADS>(p.work, blockIdx.x, sh.found, walk);
    __syncthreads();                     // `found` makes room for the scales
    auto wait_all = [&](uint64_t *bar, uint32_t parity) -> bool {
        return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_v, p.err));
    };
    // the n-th piece, once it is there
    auto piece = [&](int n, bool &ok) -> const KvPiece & {
        ok = wait_all(&sh.piece_full[n % PIECES], (n / PIECES) & 1);
        return sh.piece[n % PIECES];
    };
    auto piece_done = [&](int n) {
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.piece_empty[n % PIECES]);
    };

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::REGS[0]) : "memory");
        bool ok = true;
        if (warp == 3) {
            // ---------------- pieces, and their queries ----------------
            int n = 0, loads = 0;
            if (lane == 0) kv_leave_join(p.work, walk, p.ws, D);
            for (bool more = true; more; ++n) {
                more = walk.next(p.work);
                // Items that see no key become zeros here: the other warps get pieces with
                // blocks only.  (They look one piece ahead, and a row of empty ones longer
                // than the pieces handed out would keep each waiting for the other.)
                while (more && walk.kb0 == walk.kb1) {
                    const int first = walk.tile * p.work.tile, rows = min(p.work.tile, walk.s.packed - first);
                    for (int i = lane; i < rows * (D / 8); i += 32) {
                        const int pr = first + i / (D / 8);
                        const int r = p.work.by_group(pr), h = pr - r * p.work.group;
                        *reinterpret_cast<uint4 *>(p.out + (int64_t)(walk.s.row + r) * p.ldo +
                                                   (walk.head * p.work.group + h) * D + i % (D / 8) * 8) =
                            make_uint4(0, 0, 0, 0);
                    }
                    more = walk.next(p.work);
                }
                if (n >= PIECES && !wait_all(&sh.piece_empty[n % PIECES], ((n / PIECES) & 1) ^ 1)) break;
                KvPiece &pc = sh.piece[n % PIECES];
                if (lane == 0) {
                    if (more) {
                        walk.put(p.work, pc);
                        if (walk.s.len > p.work.cap) echo_flag_error(p.err, ECHO_ERR_PAGE);
                        if (walk.tail()) kv_leave_join(p.work, walk, p.ws, D);
                    } else {
                        pc.blocks = -1;
                    }
                    mbar_arrive(&sh.piece_full[n % PIECES]);
                }
                __syncwarp();
                if (!more) continue;
                // the queries' buffer is free once the last S of its piece before is done
                const int qb = loads % C::Q_BUFS, use = loads / C::Q_BUFS;
                if (use > 0 && !wait_all(&sh.q_empty[qb], (use - 1) & 1)) break;
                if (lane == 0) {
                    mbar_arrive_expect_tx(&sh.q_full[qb], TILES * C::ATOMS * p.tile_rows * 128);
                    const int tokens = p.work.by_group(p.tile_rows);
                    for (int t = 0; t < TILES; ++t)
                        for (int a = 0; a < C::ATOMS; ++a)
                            tma_load_3d(Qs + qb * C::Q_BUF + t * C::Q_BYTES + a * ATOM, &tm_q, &sh.q_full[qb], 64 * a,
                                        walk.head * p.work.group,
                                        walk.s.row + (walk.tile * TILES + t) * tokens);
                }
                ++loads;
            }
            // copies land before this CTA exits, whoever gives up, and when
            for (int i = max(0, loads - C::Q_BUFS); i < loads; ++i)
                mbar_land(&sh.q_full[i % C::Q_BUFS], (i / C::Q_BUFS) & 1);
        } else if (warp == 0) {
            // ---------------- keys and values, a page at a time ----------------
            const int shift = p.pool.shift, per_block = BN >> shift;
            int li = 0;                                       // copies into the ring so far
            for (int n = 0; ok; ++n) {
                const KvPiece &pc = piece(n, ok);
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
                        // d 128: a slot; 64: those of V_f and K_{f+1}
                        if (D == 128) ok = wait_all(&sh.empty[slot], ((li / RING) & 1) ^ 1);
                        else if (kv == 1) ok = wait_all(&sh.empty[((li >> 1) + 1) % 3], ((((li >> 1) + 1) / 3) & 1) ^ 1);
                        if (!ok) break;
                        uint64_t *bar = INT8 ? &sh.raw_full[slot] : li == 0 ? &sh.k_first : &sh.pair[((li - 1) >> 1) % PAIRS];
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
            // the last V has no K after it
            if (!INT8 && li > 0 && lane == 0) mbar_arrive(&sh.pair[((li - 1) >> 1) % PAIRS]);
            // copies land before this CTA exits, whoever gives up, and when
            if (INT8) {
                for (int i = max(0, li - RING); i < li; ++i) mbar_land(&sh.raw_full[i % RING], (i / RING) & 1);
            } else if (li > 0) {
                mbar_land(&sh.k_first, 0);
                for (int i = max(0, li / 2 - PAIRS); i < li / 2; ++i) mbar_land(&sh.pair[i % PAIRS], (i / PAIRS) & 1);
            }
        } else if (warp == 1) {
            // ---------------- products of both tiles ----------------
            // The whole warp runs the loop and one elected lane issues (attn_tc_kernel of
            // attention.cu).  P_t lies over the first half of S_t: MMAs of one thread run in
            // order, so S of the next block cannot overtake the P V that reads it.  A wait
            // costs about 130 cycles even when there is nothing to wait for, more than the
            // tensor cores' queue holds: three a block, the next tiles' in the window of the
            // first tile's softmax.  Whatever the loop carries comes from votes, which the
            // compiler knows to be the same in every lane; from values read from memory it
            // would move every descriptor to the uniform registers one by one.
            const bool leader = elect_one_sync();
            constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
            constexpr uint32_t LO_K = 1u << 16;
            constexpr uint32_t LO_MN = (uint32_t)(ATOM >> 4) << 16;
            const uint32_t q_lo = ((smem_u32(Qs) & 0x3FFFFu) >> 4) | LO_K;
            const uint32_t ring_lo = (smem_u32(Ring) & 0x3FFFFu) >> 4;
            auto desc = [](uint32_t lo) -> uint64_t { return ((uint64_t)DESC_HI << 32) | lo; };
            auto mma_s = [&](int t, int slot, int buf, int qb) {
                const uint32_t a_lo = q_lo + (uint32_t)(qb * (C::Q_BUF >> 4) + t * (C::Q_BYTES >> 4));
                const uint32_t b_lo = (ring_lo + (uint32_t)slot * (C::SLOT >> 4)) | LO_K;
                const uint32_t d = tmem + (uint32_t)(buf * BN);
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    const uint32_t off = (uint32_t)(((kk >> 2) * ATOM + (kk & 3) * 32) >> 4);
                    tc_mma_f16(d, desc(a_lo + off), desc(b_lo + off), C::IDESC_S, kk > 0);
                }
            };
            auto mma_pv = [&](int t, int slot, int buf, uint32_t acc0) {
                const uint32_t b_lo = (ring_lo + (uint32_t)slot * (C::SLOT >> 4)) | LO_MN;
                const uint32_t d = tmem + C::O_COL + (uint32_t)(t * D);
                const uint32_t a = tmem + (uint32_t)(buf * BN);
                tc_mma_f16_tmem_a(d, a, desc(b_lo), C::IDESC_PV, acc0);
#pragma unroll
                for (int kk = 1; kk < BN / 16; ++kk)
                    tc_mma_f16_tmem_a(d, a + 8 * kk, desc(b_lo + (uint32_t)(kk * 2048 >> 4)), C::IDESC_PV, 1u);
            };
            auto uniform = [&](int v) -> int { return (int)__ballot_sync(0xffffffffu, (v >> lane) & 1); };
            auto next2 = [](int s) { return s + 2 >= RING ? s + 2 - RING : s + 2; };
            int pr = 0;                                       // barrier of the next pair, and its parity
            uint32_t pph = 0, eph = 0;                        // and that of edges
            [[maybe_unused]] uint32_t fph = 0, qph = 0;       // of P, of Q
            auto wait_pair = [&]() -> bool {
                const bool there = wait_all(&sh.pair[pr], pph);
                if (++pr == PAIRS) { pr = 0; pph ^= 1u; }
                return there;
            };
            auto edge_go = [&]() { if (!INT8 && lane == 0) mbar_arrive(&sh.edge_go); };
            auto edge_wait = [&]() -> bool {
                if (INT8) return true;
                const bool there = wait_all(&sh.v_ok, eph);
                eph ^= 1u;
                return there;
            };
            if constexpr (D == 64) {
                // Work items k = 2 f + t (block f, tile t) in S buffer k mod 3, in the order
                //   S(0) S(1) S(2) | PV(0) S(3) | PV(1) S(4) | ...
                // S(k + 3) goes over P(k) right after P V of item k has been issued, and
                // S(k + 2), the tile's next block, is done while its softmax still works on
                // item k.  With two buffers each tile's softmax waited for its products
                // (4864 rows, 8192 keys, 8 heads of 64: 82 us, so 69); d 128, whose products
                // take twice as long, has room for two only (tensor pipe 65 % active).  S runs
                // ahead across pieces, whose queries have two buffers.  Issuing must not cost
                // more than the 1024 cycles of a block's products: a commit takes about 80
                // cycles and a wait 130, so V_f and K_{f+1} are freed by one commit, and
                // blocks without an edge have a loop of their own (without either: 103 us).
                int n_s = 0, s_left = 0, s_j = 0, s_clear = 0;   // piece that S is in, its blocks
                int ks = 0, s_bar = 0, s_blocks = 0, pairs = 0;  // slot of S's K; blocks begun, pairs seen
                bool s_end = false, edge = false;             // no more; the last block begun is an edge
                auto see_pair = [&]() -> bool {
                    if (!wait_pair()) return false;
                    if (edge) edge_go();
                    ++pairs;
                    return true;
                };
                // S of tile t of the next block: before it, what the block needs
                auto next_s = [&]() -> bool {
                    if (s_left == 0) {
                        const KvPiece &pc = piece(n_s, ok);
                        if (!ok) return false;
                        s_left = uniform(pc.blocks);
                        s_clear = uniform(kv_clear(pc));
                        s_j = 0;
                        s_end = s_left < 0;
                        if (s_end) return true;
                        if (!wait_all(&sh.q_full[n_s & 1], (n_s >> 1) & 1)) return false;
                        ++n_s;
                    }
                    // K_f comes with V_{f-1}
                    if (!(s_blocks == 0 ? wait_all(&sh.k_first, 0) : see_pair())) return false;
                    ++s_blocks;
                    edge = s_j >= s_clear;
                    return true;
                };
                auto issue_s = [&](int t, int buf) {
                    const int qb = (n_s - 1) & 1;
                    if (leader) {
                        mma_s(t, ks, buf, qb);
                        tc_commit(&sh.s_full[s_bar]);
                        if (t == 1) {
                            if (s_blocks == 1) tc_commit(&sh.empty[0]);   // K_0
                            if (s_left == 1) tc_commit(&sh.q_empty[qb]);
                        }
                    }
                    __syncwarp();
                    if (++s_bar == C::S_BARS) s_bar = 0;
                    if (t == 1) {
                        ks = next2(ks);
                        --s_left;
                        ++s_j;
                    }
                };
                int n = 0, f = 0, j = 0, nb = 0, nclear = 0;  // piece and block that P V is in
                int vs = 1, rel = 1, t = 1, buf = 0;          // rel: of V_f and K_{f+1}
                uint32_t pbuf = 0;                            // parity of the S buffers' P
                // two S before the first P V; from then on P V of an item, S of the third after it
                for (int item = -3; ok; ++item) {
                    if (item >= 0) {
                        if (t == 1) {                         // next: the tile 0 of a block
                            if (j == nb) {
                                const KvPiece &pc = piece(n, ok);
                                if (!ok) break;
                                nb = uniform(pc.blocks);
                                nclear = uniform(kv_clear(pc));
                                if (nb < 0) break;
                                piece_done(n++);              // S has been here
                                j = 0;
                            }
                            // blocks without an edge, S in the same piece
                            const int plain = min(nclear - 1, nb - 2);
                            if (j < plain) {
                                const int some = plain - j, qb = (n_s - 1) & 1;
                                for (; ok && j < plain; ++j) {
                                    const int buf1 = buf + 1 == C::S_BUFS ? 0 : buf + 1;
                                    ok = wait_all(&sh.p_full[buf], pbuf);
                                    if (!ok) break;
                                    tc_fence_after();
                                    if (leader) {
                                        mma_pv(0, vs, buf, j > 0 ? 1u : 0u);
                                        mma_s(1, ks, buf, qb);
                                        tc_commit(&sh.s_full[s_bar]);
                                    }
                                    __syncwarp();
                                    if (buf == 2) pbuf ^= 1u;
                                    ks = next2(ks);
                                    if (++s_bar == C::S_BARS) s_bar = 0;
                                    ok = wait_pair() && wait_all(&sh.p_full[buf1], pbuf);
                                    if (!ok) break;
                                    tc_fence_after();
                                    if (leader) {
                                        mma_pv(1, vs, buf1, j > 0 ? 1u : 0u);
                                        tc_commit(&sh.empty[rel]);
                                        mma_s(0, ks, buf1, qb);
                                        tc_commit(&sh.s_full[s_bar]);
                                    }
                                    __syncwarp();
                                    if (buf1 == 2) pbuf ^= 1u;
                                    if (++s_bar == C::S_BARS) s_bar = 0;
                                    vs = next2(vs);
                                    if (++rel == 3) rel = 0;
                                    buf = buf1 + 1 == C::S_BUFS ? 0 : buf1 + 1;
                                }
                                if (!ok) break;
                                f += some;
                                pairs += some;
                                s_left -= some;
                                s_j += some;
                                s_blocks += some;
                                edge = s_j >= s_clear;
                            }
                            if (pairs <= f) ok = see_pair();  // the last block's V comes alone
                            if (ok && j >= nclear) ok = edge_wait();
                            if (!ok) break;
                        }
                        t ^= 1;
                        ok = wait_all(&sh.p_full[buf], pbuf);
                        if (!ok) break;
                        tc_fence_after();
                        if (leader) {
                            mma_pv(t, vs, buf, j > 0 ? 1u : 0u);
                            if (t == 1) tc_commit(&sh.empty[rel]);
                            if (j == nb - 1) tc_commit(&sh.pv_done[t]);
                        }
                        __syncwarp();
                        if (t == 1) {
                            vs = next2(vs);
                            if (++rel == 3) rel = 0;
                            ++j;
                            ++f;
                        }
                    }
                    const int ts = (item + 3) & 1;
                    if (!s_end && ts == 0) ok = next_s();
                    if (!ok) break;
                    if (!s_end) {
                        tc_fence_after();
                        issue_s(ts, buf);
                    }
                    if (++buf == C::S_BUFS) {
                        buf = 0;
                        if (item >= 0) pbuf ^= 1u;
                    }
                }
            } else {
                int n = 0;                                        // pieces taken
                int blocks = 0, clear = 0;                        // of the piece that is there
                // the next piece; none: blocks 0
                auto next_piece = [&]() {
                    const KvPiece &pc = piece(n, ok);
                    blocks = 0;
                    if (!ok) return;
                    blocks = max(uniform(pc.blocks), 0);
                    clear = uniform(kv_clear(pc));
                    if (blocks > 0) piece_done(n++);
                };
                int vs = 1, ks = 2;                               // slots of V_f and K_{f+1}
                next_piece();
                if (ok && blocks > 0 && (ok = wait_all(&sh.q_full[0], 0) && wait_all(&sh.k_first, 0))) {
                    tc_fence_after();
                    if (leader) {
                        mma_s(0, 0, 0, 0);
                        tc_commit(&sh.s_full[0]);
                        mma_s(1, 0, 1, 0);
                        tc_commit(&sh.s_full[1]);
                        tc_commit(&sh.empty[0]);
                        if (blocks == 1) tc_commit(&sh.q_empty[0]);
                    }
                    __syncwarp();
                    ok = wait_pair();
                    if (clear == 0) edge_go();
                }
                while (ok && blocks > 0) {
                    const int nb = blocks, nclear = clear;
                    // all blocks but the last: here V_f and K_{f+1} are there.  EDGE: some row may
                    // not see the block, or the next one, whole, or the next one is the last
                    auto block = [&](int j, auto EDGE) -> bool {
                        if (EDGE && j >= nclear && !edge_wait()) return false;
                        if (!wait_all(&sh.p_full[0], fph)) return false;
                        tc_fence_after();
                        if (leader) {
                            mma_pv(0, vs, 0, j > 0 ? 1u : 0u);
                            mma_s(0, ks, 0, 0);
                            tc_commit(&sh.s_full[0]);
                        }
                        __syncwarp();
                        if (!wait_all(&sh.p_full[1], fph)) return false;
                        tc_fence_after();
                        if (leader) {
                            mma_pv(1, vs, 1, j > 0 ? 1u : 0u);
                            tc_commit(&sh.empty[vs]);
                            mma_s(1, ks, 1, 0);
                            tc_commit(&sh.s_full[1]);
                            tc_commit(&sh.empty[ks]);
                            if (EDGE && j == nb - 2) tc_commit(&sh.q_empty[0]);
                        }
                        __syncwarp();
                        vs = next2(vs);
                        ks = next2(ks);
                        fph ^= 1u;
                        if (!wait_pair()) return false;
                        if (EDGE && j + 1 >= nclear) edge_go();
                        return true;
                    };
                    const int plain = min(nclear - 1, nb - 2);
                    int j = 0;
                    for (; ok && j < plain; ++j) ok = block(j, std::false_type());
                    for (; ok && j < nb - 1; ++j) ok = block(j, std::true_type());
                    if (!ok) break;
                    // the last block, and the next piece's first S
                    const uint32_t acc = nb > 1 ? 1u : 0u;
                    if (nclear < nb && !edge_wait()) { ok = false; break; }
                    next_piece();
                    if (!ok || !wait_all(&sh.p_full[0], fph)) { ok = false; break; }
                    tc_fence_after();
                    if (leader) {
                        mma_pv(0, vs, 0, acc);
                        tc_commit(&sh.pv_done[0]);
                    }
                    __syncwarp();
                    if (blocks > 0) {
                        qph ^= 1u;
                        if (!wait_all(&sh.q_full[0], qph)) { ok = false; break; }
                        tc_fence_after();
                        if (leader) {
                            mma_s(0, ks, 0, 0);
                            tc_commit(&sh.s_full[0]);
                        }
                        __syncwarp();
                    }
                    if (!wait_all(&sh.p_full[1], fph)) { ok = false; break; }
                    tc_fence_after();
                    if (leader) {
                        mma_pv(1, vs, 1, acc);
                        tc_commit(&sh.empty[vs]);
                        tc_commit(&sh.pv_done[1]);
                        if (blocks > 0) {
                            mma_s(1, ks, 1, 0);
                            tc_commit(&sh.s_full[1]);
                            tc_commit(&sh.empty[ks]);
                            if (blocks == 1) tc_commit(&sh.q_empty[0]);
                        }
                    }
                    __syncwarp();
                    vs = next2(vs);
                    ks = next2(ks);
                    fph ^= 1u;
                    if (blocks > 0) {
                        ok = wait_pair();
                        if (ok && clear == 0) edge_go();
                    }
                }
            }
            if (!ok && leader) {   // the MMAs already issued, before tensor memory is freed
                tc_commit(&sh.drain);
                mbar_land(&sh.drain, 0);
            }
            __syncwarp();
        }
    } else if (warp < C::SOFT0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::REGS[1]) : "memory");
        bool ok = true;
        int f = 0;                                            // block
        if constexpr (!INT8) {
            // ---------------- values that no row may use, cleared ----------------
            int edge = 0;
            for (int n = 0; ok; ++n) {
                const KvPiece &pc = piece(n, ok);
                if (!ok || pc.blocks < 0) break;
                const int blocks = pc.blocks, clear = kv_clear(pc), keys = pc.keys - pc.kb0 * BN;
                piece_done(n);
                f += clear;
                for (int j = clear; j < blocks; ++j, ++f, ++edge) {
                    // from the warp that issues the products: it has seen V_f's copy
                    const int slot = (2 * f + 1) % RING;
                    ok = wait_all(&sh.edge_go, edge & 1);
                    if (!ok) break;
                    {
                        const int valid = keys - j * BN;
                        const int r0 = (warp - 4) * 32;       // this warp's keys
                        uint32_t spoilt = 0;
#pragma unroll 4
                        for (int i = lane; i < 32 * C::ATOMS * 8; i += 32) {
                            const int r = r0 + ((i >> 3) & 31), a = i >> 8;
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
                                if (r < valid) spoilt |= 1u << (r & 31);
                            }
                        }
                        spoilt = __reduce_or_sync(0xffffffffu, spoilt);
                        if (lane == 0) sh.spoilt[edge % SPOILT][warp - 4] = spoilt;
                        fence_proxy_async_smem();
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.v_ok);
                }
            }
        } else {
        // ---------------- codes to bf16, a key per thread ----------------
        const int r = threadIdx.x & 127;                      // key of the block
        for (int n = 0; ok; ++n) {
            const KvPiece &pc = piece(n, ok);
            if (ok && pc.blocks < 0 && f > 0 && lane == 0)    // the last V has no K after it
                mbar_arrive(&sh.pair[(f - 1) % PAIRS]);
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
                    float ks = 0.f, vs = 0.f;
                    if (kv == 0) {
                        const float *sc = reinterpret_cast<const float *>(tile + (r & ~31) * 128) + lane;
                        ks = sc[0];
                        vs = sc[32];
                        __syncwarp();                         // read before the rows are written
                        if (!(fabsf(vs) < INFINITY)) ks = NAN, vs = 0.f;
                        if (kb * BN + r >= keys) ks = vs = 0.f;   // slots past the end: anything
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
                            const uint32_t w[4] = {kv_flip(in[c].x), kv_flip(in[c].y), kv_flip(in[c].z), kv_flip(in[c].w)};
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
                    if (lane == 0) mbar_arrive(li == 0 ? &sh.k_first : &sh.pair[((li - 1) >> 1) % PAIRS]);
                    if (kv == 0) {                            // of block f - 2: done with by now
                        ok = wait_all(&sh.sc_empty[f & 1], ((f >> 1) & 1) ^ 1);
                        if (!ok) break;
                        sh.scales[f & 1][0][r % (INT8 ? BN : 1)] = ks * p.scale_log2;
                        sh.scales[f & 1][1][r % (INT8 ? BN : 1)] = vs * kCodeUnit;
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&sh.sc_full[f & 1]);
                    }
                }
            }
        }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::REGS[2]) : "memory");
        // ---------------- softmax and output of tile t, a row per thread ----------------
        const int t = (warp - C::SOFT0) >> 2, quad = warp & 3;
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        const uint32_t o_at = tmem + lane_base + C::O_COL + (uint32_t)(t * D);
        int s_bar = t;                                        // of S of this block, and its parity
        uint32_t sph = 0;
        const int row = quad * 32 + lane;                     // of the tile
        bool ok = true;
        int f = 0, edge = 0;
        for (int n = 0; ok; ++n) {
            const KvPiece &pc = piece(n, ok);
            if (!ok || pc.blocks < 0) break;
            const int pr = (pc.tile * TILES + t) * p.tile_rows + row;        // packed row
            const bool real = row < p.tile_rows && pr < pc.packed;
            int lim = pc.keys;                                // keys that the row sees
            if (real) {
                KvSeq s;
                s.len = pc.len;
                s.shift = pc.shift;
                lim = s.top(p.work, pc.row + p.work.by_group(pr));
            }
            const int warp_low = __reduce_min_sync(0xffffffffu, lim);
            const int kb0 = pc.kb0, blocks = pc.blocks, clear = kv_clear(pc);
            // Rows of a lane: its own, a whole row of S per thread.  int8: rows gq + 8 x of the
            // warp's 32, every fourth pair of columns, as the fragments of a product lie, so
            // that a lane needs only a quarter of the scales (a whole row per thread loads all
            // 256 of a block: 487 us where this took 450, 4864 rows over 32768 keys, 8 heads of 128)
            constexpr int NX = INT8 ? 4 : 1;
            const int gq = lane >> 2, tq = lane & 3;
            float m[NX], l[NX];
            int seen[NX];                                     // keys that the rows see
#pragma unroll
            for (int x = 0; x < NX; ++x) {
                m[x] = -FLT_MAX;
                l[x] = 0.f;
                seen[x] = INT8 ? __shfl_sync(0xffffffffu, lim, gq + 8 * x) : lim;
            }
            // the value of this thread's own row
            auto own = [&](const float *v) -> float {
                if constexpr (!INT8) return v[0];
                float r = 0.f;
#pragma unroll
                for (int x = 0; x < NX; ++x) {
                    const float y = __shfl_sync(0xffffffffu, v[x], (lane & 7) * 4);
                    if (lane >> 3 == x) r = y;
                }
                return r;
            };
            for (int j = 0; j < blocks; ++j, ++f) {
                ok = wait_all(&sh.s_full[s_bar], sph);
                if (!ok) break;
                tc_fence_after();
                const int buf = s_bar >= C::S_BUFS ? s_bar - C::S_BUFS : s_bar;
                const uint32_t s_at = tmem + lane_base + (uint32_t)(buf * BN);
                const int key0 = (kb0 + j) * BN;
                if constexpr (INT8) {
                    ok = wait_all(&sh.sc_full[f & 1], (f >> 1) & 1);
                    if (!ok) break;
                }
                const bool edge_block = key0 + BN > warp_low;
                // the scores of 32 keys at a time, the next ones on their way
                float sv[2][32];
                auto load32 = [&](int c) {
                    uint32_t *to = reinterpret_cast<uint32_t *>(sv[c & 1]);
                    if constexpr (INT8) {
                        tmem_ld_frag32(s_at + 32 * c, to);
                        tmem_ld_frag32(s_at + 32 * c + (16u << 16), to + 16);
                    } else {
                        tmem_ld32(s_at + 32 * c, to);
                    }
                };
                auto each32 = [&](auto f32) {
                    load32(0);
#pragma unroll
                    for (int c = 0; c < BN / 32; ++c) {
                        tmem_ld_wait();
                        if (c + 1 < BN / 32) load32(c + 1);
                        f32(c, sv[c & 1]);
                    }
                };
                // pair i of the 32 keys' in v[2 i], v[2 i + 1]: whose row, and its first key;
                // the scales of keys 2 k and 2 k + 1 of the block
                auto row_of = [](int i) { return INT8 ? 2 * (i >> 3) + (i & 1) : 0; };
                auto key_of = [&](int i) { return INT8 ? 8 * ((i >> 1) & 3) + 2 * tq : 2 * i; };
                auto scale2 = [&](int kv, int key) -> uint64_t {
                    const float2 s2 = *reinterpret_cast<const float2 *>(&sh.scales[INT8 ? f & 1 : 0][kv][key]);
                    return f2_pack(s2.x, s2.y);
                };
                const uint64_t unit2 = f2_pack(p.scale_log2, p.scale_log2);
                // -inf where the row does not see the key.  int8: after the keys' scales, which
                // may be 0 (elsewhere they are part of the exponent's product)
                auto mask32 = [&](int c, float *v) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        if constexpr (INT8)
                            f2_unpack(f2_mul(f2_pack(v[2 * i], v[2 * i + 1]), scale2(0, 32 * c + key_of(i))), v[2 * i], v[2 * i + 1]);
                        if (edge_block) {
                            const int k = key0 + 32 * c + key_of(i);
                            if (k >= seen[row_of(i)]) v[2 * i] = -INFINITY;
                            if (k + 1 >= seen[row_of(i)]) v[2 * i + 1] = -INFINITY;
                        }
                    }
                };
                // the rows' largest scores of the block, in the exponent of two
                auto row_max = [&](float *mx) {
#pragma unroll
                    for (int x = 0; x < NX; ++x) mx[x] = -INFINITY;
                    each32([&](int c, float *v) {
                        mask32(c, v);
#pragma unroll
                        for (int i = 0; i < 16; ++i) mx[row_of(i)] = fmax3(mx[row_of(i)], v[2 * i], v[2 * i + 1]);
                    });
#pragma unroll
                    for (int x = 0; x < NX; ++x) {
                        if constexpr (INT8) {
                            mx[x] = fmaxf(mx[x], __shfl_xor_sync(0xffffffffu, mx[x], 1));
                            mx[x] = fmaxf(mx[x], __shfl_xor_sync(0xffffffffu, mx[x], 2));
                        } else {
                            mx[x] *= p.scale_log2;
                        }
                    }
                };
                // P = 2^(s - m) on fp32 pairs, times the values' scales, in bf16 pairs; this
                // lane's part of the rows' sums of 2^(s - m); whether one is above 2^64 or NaN
                uint32_t pk[BN / 2];
                float bsum[NX];
                auto exp_pass = [&](auto EDGE) -> bool {
                    uint64_t negm2[NX], acc2[4];
#pragma unroll
                    for (int x = 0; x < NX; ++x) negm2[x] = f2_pack(-m[x], -m[x]);
#pragma unroll
                    for (int x = 0; x < 4; ++x) acc2[x] = 0ull;
                    each32([&](int c, float *v) {
                        if constexpr (EDGE) mask32(c, v);
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const uint64_t s2 = f2_pack(v[2 * i], v[2 * i + 1]);
                            uint64_t k2 = unit2;
                            if constexpr (INT8 && !EDGE) k2 = scale2(0, 32 * c + key_of(i));
                            float x0, x1;
                            if constexpr (INT8 && EDGE) f2_unpack(f2_add(s2, negm2[row_of(i)]), x0, x1);
                            else f2_unpack(f2_fma(s2, k2, negm2[row_of(i)]), x0, x1);
                            float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
                            const int to = INT8 ? row_of(i) : i & 3;
                            acc2[to] = f2_add(acc2[to], f2_pack(p0, p1));
                            if constexpr (INT8) {
                                f2_unpack(f2_mul(f2_pack(p0, p1), scale2(1, 32 * c + key_of(i))), p0, p1);
                                pk[32 * (i >> 3) + 2 * (4 * c + ((i >> 1) & 3)) + (i & 1)] = pack_bf16(p0, p1);
                            } else {
                                pk[16 * c + i] = pack_bf16(p0, p1);
                            }
                        }
                    });
                    bool high = false;
                    if constexpr (!INT8) acc2[0] = f2_add(f2_add(acc2[0], acc2[1]), f2_add(acc2[2], acc2[3]));
#pragma unroll
                    for (int x = 0; x < NX; ++x) {
                        float a0, a1;
                        f2_unpack(acc2[x], a0, a1);
                        bsum[x] = a0 + a1;
                        high |= !(bsum[x] <= 1.8446744e19f);
                    }
                    return __any_sync(0xffffffffu, high);
                };
                float mx[NX];
                // a first block that shows the row no key leaves the maximum at the lowest
                // number: P is 0 there, and the first finite score overflows and brings its own
                if (j == 0) {
                    row_max(mx);
#pragma unroll
                    for (int x = 0; x < NX; ++x) m[x] = fmaxf(mx[x], -FLT_MAX);
                }
                if (edge_block ? exp_pass(std::true_type()) : exp_pass(std::false_type())) {
                    row_max(mx);
                    float a[NX];
#pragma unroll
                    for (int x = 0; x < NX; ++x) {
                        const float high = fmaxf(m[x], mx[x]);
                        a[x] = ex2_approx(m[x] - high);
                        l[x] *= a[x];
                        m[x] = high;
                    }
                    const float alpha = own(a);
                    if (j > 0) {
                        // two S buffers: S of this block completed after P V of the one before
                        // (three: the next item's S did, or for the piece's last P V, tile 0's)
                        if constexpr (D == 64) {
                            const int next = 2 * f + t + 1;
                            ok = t == 1 && j == blocks - 1 ? wait_all(&sh.pv_done[0], n & 1)
                                                           : wait_all(&sh.s_full[next % 6], (next / 6) & 1);
                            if (!ok) break;
                            tc_fence_after();
                        }
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
                    if (edge_block) exp_pass(std::true_type());
                    else exp_pass(std::false_type());
                }
#pragma unroll
                for (int x = 0; x < NX; ++x) l[x] += bsum[x];
                if constexpr (INT8) {
                    tmem_st_frag64(s_at, pk);
                    tmem_st_frag64(s_at + (16u << 16), pk + 32);
                } else {
                    tmem_st32(s_at, pk);
                    tmem_st32(s_at + 32, pk + 32);
                }
                tmem_st_wait();
                if (!INT8 && j >= clear) {                      // keys whose values are not finite
                    ok = wait_all(&sh.v_ok, edge & 1);
                    if (!ok) break;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int some = lim - key0 - 32 * e;
                        const uint32_t mask = some >= 32 ? 0xffffffffu : some > 0 ? (1u << some) - 1u : 0u;
                        if (sh.spoilt[edge % SPOILT][e] & mask) l[0] = NAN;
                    }
                    ++edge;
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&sh.p_full[buf]);
                    if constexpr (INT8) mbar_arrive(&sh.sc_empty[f & 1]);
                }
                s_bar += TILES;
                if (s_bar >= C::S_BARS) {
                    s_bar = t;
                    sph ^= 1u;
                }
            }
            if (!ok) break;
            ok = wait_all(&sh.pv_done[t], n & 1);
            if (!ok) break;
            tc_fence_after();
            if constexpr (INT8) {
#pragma unroll
                for (int x = 0; x < NX; ++x) {
                    l[x] += __shfl_xor_sync(0xffffffffu, l[x], 1);
                    l[x] += __shfl_xor_sync(0xffffffffu, l[x], 2);
                }
            }
            const bool whole = pc.whole;
            const float m_row = own(m), l_row = own(l);
            const float inv = l_row == 0.f ? 0.f : 1.f / l_row;  // no key: zeros
            __nv_bfloat16 *dst = nullptr;
            float *part = nullptr;
            if (real) {
                const int g = p.work.group, r = p.work.by_group(pr);
                dst = p.out + (int64_t)(pc.row + r) * p.ldo + (pc.head * g + pr - r * g) * D;
            }
            const int slot_row = t * p.tile_rows + row;
            if (!whole) {
                part = kv_slot(p.ws, blockIdx.x, pc.tail, SLOT_ROWS, D);
                if (real) *reinterpret_cast<float2 *>(part + SLOT_ROWS * D + 2 * slot_row) = make_float2(m_row, l_row);
                part += (int64_t)slot_row * D;
            }
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                uint32_t o[32];
                tmem_ld32(o_at + 32 * c, o);
                tmem_ld_wait();
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
    p.work = echo::kv_work(a, TILES * p.tile_rows, SLOT_ROWS, 7, echo::num_sms(), kWholeKeys);
    p.out = static_cast<__nv_bfloat16 *>(a.out);
    p.ws = static_cast<float *>(a.ws);
    p.ldo = a.ldo;
    p.scale_log2 = 1.4426950408889634f / sqrtf((float)D) * (INT8 ? kCodeUnit : 1.f);
    p.err = echo::device_error_ptr();
    cudaError_t launched;
    {
        echo::LaunchScope ls(ECHO_K_KV_ATTENTION, a.batch->n_rows, (int64_t)a.Hq * D, a.batch->n_seqs, st);
        launched = echo::launch_chained(kv_chunk_kernel<INT8, D>, dim3(p.work.workers), dim3(C::THREADS), SMEM, st, tq, tk, p);
    }
    if (launched == cudaSuccess) echo::launch_kv_join(a, p.work, st);   // it needs what the kernel leaves
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
