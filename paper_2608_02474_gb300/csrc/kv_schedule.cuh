// How the work of one attention call over the paged cache is divided between CTAs
// ("workers"), on the device, since the sequences' lengths are known only there.
//
// Items: (sequence, key/value head, row tile).  The Hq / H query heads that share a
// key/value head are packed with the rows, packed row = row * group + head of the group,
// and a tile is `tile` of them, so that keys and values are read once for all.  An item
// costs kFixedUnits + (its key blocks) units, and every worker gets the same sum of units.
//
// As many items as every worker can take whole go round first, in their order: worker c of
// G takes W of them from item W c on.  The units of the items left over are dealt out so
// that the workers' sums come out even, in one row, each worker's next to the one's before
// and no worker between two others without any (the joining kernel relies on it).
// An item that crosses a boundary there is done in pieces: each worker leaves its piece's
// sums in the workspace, and the joining kernel adds them up.  A worker has at most one
// piece with an item's last keys but not its first (an item that it begins, and others go
// on with), and one other: two slots of workspace each.
//
// The whole items of all workers begin together, and the tiles of a head run through its
// keys in step, so that a key block is read from memory once and from the L2 by the
// others.  For the same reason the worker that goes on with an item takes its first keys.
// 1560 rows over 32760 keys (40 heads of 128, bf16): one row of all items, each worker's
// share in the items' order 768 us; whole items first, and the first keys to the later
// worker 695; as it is 662.
#pragma once

#include "kv_pages.cuh"

// Division of 0 .. 2^31 - 1 by a number known to the host, as a product: with s = ceil(log2 d)
// and m = ceil(2^(31 + s) / d), m d exceeds 2^(31 + s) by less than 2^s, so that n m / 2^(31 + s)
// exceeds n / d by less than 1 / d.
struct KvDiv {
    uint32_t m;
    int s, d;
    explicit KvDiv(int by = 1) : m(0), s(0), d(by) {
        while ((1ll << s) < by) ++s;
        if (s > 0) m = (uint32_t)(((1ull << (31 + s)) + by - 1) / by);
    }
    ECHO_DEV int operator()(int n) const { return s == 0 ? n : (int)(__umulhi((uint32_t)n, m) >> (s - 1)); }
};
// as 32-bit numbers where they are: a division of 64 bits takes several hundred cycles
ECHO_DEV int64_t kv_div64(int64_t a, int64_t b) {
    return (uint64_t)(a | b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

struct KvWork {
    KvBatch b;
    int H, group, causal_block;
    KvDiv by_group, by_tile, by_block;
    int tile, slot_rows;   // packed rows of a tile, and rows of a workspace slot
    int cap;               // positions that a table row covers
    int block_shift;       // keys of a block, as a power of two
    int workers;
    int split;             // 0: items are not divided; each goes to the worker of its first unit
};

constexpr int kFixedUnits = 2;   // set-up and end of a piece, in key-block times
constexpr int kLeast = 4;        // the fewest units for a worker
constexpr int kMostKeys = INT32_MAX / 128 * 128;   // of a sequence: whole blocks and pages in 31 bits

struct KvSeq {             // one sequence of the batch
    int row, packed, len;  // its first row, its packed rows, its length
    int64_t shift;         // position of row r: shift + r
    ECHO_DEV void load(const KvWork &w, int seq) {
        const int a = min(max(w.b.row0[seq], 0), w.b.n_rows), e = w.b.row0[seq + 1];
        row = a;
        packed = max(min(e, w.b.n_rows) - a, 0) * w.group;
        len = max(w.b.len[seq], 0);
        shift = (int64_t)len - e;
    }
    ECHO_DEV int tiles(const KvWork &w) const { return w.by_tile(packed + w.tile - 1); }
    // keys that row r sees
    ECHO_DEV int top(const KvWork &w, int r) const {
        if (w.causal_block == 0) return min(len, w.cap);
        const int64_t p = shift + r;
        if (p < 0) return 0;
        const unsigned i = (unsigned)w.by_block((int)min(p, (int64_t)INT32_MAX));
        return (int)min((unsigned)min(len, w.cap), (i + 1u) * (unsigned)w.causal_block);
    }
    // keys that any row of tile t sees: those of its last row
    ECHO_DEV int keys(const KvWork &w, int t) const {
        const int last = min((t + 1) * w.tile, packed) - 1;
        return top(w, row + w.by_group(last));
    }
    ECHO_DEV int blocks(const KvWork &w, int t) const {
        return (keys(w, t) + (1 << w.block_shift) - 1) >> w.block_shift;
    }
};

// One piece of an item, as the warps of a CTA hand it on.
struct KvPiece {
    int64_t shift;           // KvSeq::shift
    int blocks;              // key blocks from kb0 on; < 0: no more pieces
    int kb0, keys;           // keys that any row of the tile sees
    int low;                 // keys that every row sees
    int row, packed, len, head, tile, seq;
    int whole, tail;         // all of the item's keys; or the last of them
};

// A worker's walk over its pieces: the whole items of the first round, the whole ones of its
// share of the others, and then the piece that it takes over from the worker before and the
// one that the worker after goes on with.
struct KvWalk {
    KvSeq s;
    int seq, head, tile;      // of the current piece's item
    int kb0, kb1, nb;         // its key blocks, and the item's
    int64_t start, end;       // the worker's units of the items left over
    struct Item {
        int seq, head, tile;
        int64_t at;           // its first unit
    } round, here, first;     // the next of the first round; of the others; the one that holds `start`
    int left;                 // of the first round
    int64_t from;             // the first unit of the current piece's item
    int stage;                // 0: whole items, 1: the first, 2: the last, 3: none
    bool begun;               // `start` lies inside an item

    // key blocks of an item (units from `from`) that the units before `unit` pay for, the
    // last ones first
    static ECHO_DEV int paid(int64_t unit, int64_t from, int nb) {
        return (int)min(max(unit - from - kFixedUnits, (int64_t)0), (int64_t)nb);
    }
    ECHO_DEV bool whole() const { return kb0 == 0 && kb1 == nb; }
    ECHO_DEV bool tail() const { return kb1 == nb && kb0 > 0; }

    ECHO_DEV void item(const KvWork &w, const Item &it) {
        if (it.seq != seq) s.load(w, seq = it.seq);
        head = it.head;
        tile = it.tile;
        from = it.at;
        nb = s.blocks(w, tile);
    }
    ECHO_DEV void advance(const KvWork &w, Item &it) {       // past `it`, which is the current item
        it.at += kFixedUnits + nb;
        if (++it.tile == s.tiles(w)) {
            it.tile = 0;
            if (++it.head == w.H) {
                it.head = 0;
                ++it.seq;
            }
        }
    }
    // `it`, or the first one of a later sequence that has any; false past the last
    ECHO_DEV bool settle(const KvWork &w, Item &it) {
        for (; it.seq < w.b.n_seqs; ++it.seq) {
            if (it.seq != seq) s.load(w, seq = it.seq);
            if (s.packed > 0) {
                item(w, it);
                return true;
            }
        }
        return false;
    }
    // the next piece that has something to do; false at the end
    ECHO_DEV bool next(const KvWork &w) {
        if (left > 0) {
            --left;
            settle(w, round);
            kb0 = 0;
            kb1 = nb;
            advance(w, round);
            return true;
        }
        if (stage == 0) {
            if (here.at < end && settle(w, here)) {
                if (!w.split || here.at + kFixedUnits + nb <= end) {
                    kb0 = 0;
                    kb1 = nb;
                    advance(w, here);
                    return true;
                }
            } else {
                here.seq = w.b.n_seqs;             // no last piece
            }
            stage = 1;
        }
        if (stage == 1) {
            stage = 2;
            if (begun) {
                item(w, first);
                kb1 = nb - paid(start, first.at, nb);
                kb0 = nb - paid(end, first.at, nb);
                if (kb0 < kb1) return true;
            }
        }
        if (stage == 2) {
            stage = 3;
            if (here.seq < w.b.n_seqs) {
                item(w, here);
                kb1 = nb;
                kb0 = nb - paid(end, here.at, nb);
                if (kb0 < kb1 || nb == 0) return true;
            }
        }
        kb0 = kb1 = 0;
        return false;
    }
    ECHO_DEV void put(const KvWork &w, KvPiece &pc) const {
        pc.shift = s.shift;
        pc.blocks = kb1 - kb0;
        pc.kb0 = kb0;
        pc.keys = s.keys(w, tile);
        pc.low = min(pc.keys, s.top(w, s.row + w.by_group(tile * w.tile)));
        pc.row = s.row;
        pc.packed = s.packed;
        pc.len = s.len;
        pc.head = head;
        pc.tile = tile;
        pc.seq = seq;
        pc.whole = whole();
        pc.tail = tail();
    }
};

// What the threads of a block find together.
struct KvFound {
    int64_t units[32];           // of the warps' sequences, one head each
    int items[32], most[32];     // items; the most units of one
    int64_t at[3];               // the first units of items
    KvWalk::Item begin;
    int64_t base, per_head;
    int seq;
};

// The walk of `worker`.  Called by every thread of the block.  Thread t looks at sequences
// [t per, (t + 1) per), or a warp at each where there are no more sequences than warps (a
// long chunk has many tiles).
template <int THREADS>
ECHO_DEV void kv_find(const KvWork &w, int worker, KvFound &sh, KvWalk &walk) {
    constexpr int WARPS = THREADS / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool by_warp = w.b.n_seqs <= WARPS;
    const int per = by_warp ? 1 : (w.b.n_seqs + THREADS - 1) / THREADS;
    const int b0 = by_warp ? warp : (int)threadIdx.x * per;
    const int b1 = min(b0 + per, w.b.n_seqs);
    // units of a sequence's first n tiles: by_warp this lane's share of them
    auto units_of = [&](int seq, int n, int *most) -> int64_t {
        KvSeq s;
        s.load(w, seq);
        int64_t u = 0;
        const int tiles = min(s.tiles(w), n);
        for (int t = by_warp ? lane : 0; t < tiles; t += by_warp ? 32 : 1) {
            const int v = kFixedUnits + s.blocks(w, t);
            u += v;
            *most = max(*most, v);
        }
        return u;
    };
    auto scan = [&](auto v) {                                       // inclusive, over the warp
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const auto x = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += x;
        }
        return v;
    };
    int64_t mine = 0;                                               // of one head
    int items = 0, most = 0;
    for (int i = b0; i < b1; ++i) {
        mine += units_of(i, INT32_MAX, &most);
        KvSeq s;
        s.load(w, i);
        if (!by_warp || lane == 0) items += s.tiles(w) * w.H;
    }
    const int64_t incl = scan(mine);
    const int incl_items = scan(items);
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 31) {
        sh.units[warp] = incl * w.H;
        sh.items[warp] = incl_items;
        sh.most[warp] = most;
    }
    if (threadIdx.x == 0) sh.seq = -1;
    __syncthreads();
    int64_t before = 0, total = 0;   // units of the earlier warps; of all
    int before_items = 0, all_items = 0;
    most = 1;
    for (int i = 0; i < WARPS; ++i) {
        const int64_t v = sh.units[i];
        if (i < warp) {
            before += v;
            before_items += sh.items[i];
        }
        total += v;
        all_items += sh.items[i];
        most = max(most, sh.most[i]);
    }
    const int64_t want = total / kLeast + 1;
    const int G = want < w.workers ? (int)want : w.workers;
    const int64_t per_worker = kv_div64(total, G);
    const unsigned rest = (unsigned)(total - per_worker * G);       // < G, a few hundred
    auto even = [&](int c) -> int64_t { return c < G ? per_worker * c + min((unsigned)c, rest) : total; };
    // Items of a worker.  Every worker keeps a unit of those left over, since the joining kernel
    // takes the pieces of an item from workers that follow one another.  Where all items have
    // the same units, the ones without any come after the last unit.
    int64_t round = w.split && G == w.workers ? kv_div64(per_worker, most) : 0;
    if (round > 0 && round * most == per_worker && total != (int64_t)all_items * most) --round;
    walk.start = even(worker);
    walk.end = even(worker + 1);
    walk.left = (int)round;
    if (round > 0) {
        // first units of this worker's first item of the round, of the next worker's, and of
        // the first item left over
        if (threadIdx.x < 3) sh.at[threadIdx.x] = total;
        __syncthreads();
        for (int q = 0; q < 3; ++q) {
            const int64_t at = round * (q == 0 ? worker : q == 1 ? worker + 1 : G);
            int64_t u = by_warp ? before : before + (incl - mine) * w.H;
            int64_t i0 = by_warp ? before_items : before_items + incl_items - items;
            for (int i = b0; i < b1; ++i) {
                KvSeq s;
                s.load(w, i);
                const int tiles = s.tiles(w), n = tiles * w.H;
                if (at >= i0 && at < i0 + n) {
                    const int head = (int)(at - i0) / tiles, tile = (int)(at - i0) % tiles;
                    int none = 0;
                    int64_t all = units_of(i, INT32_MAX, &none), part = units_of(i, tile, &none);
                    if (by_warp) {
                        all = __shfl_sync(0xffffffffu, scan(all), 31);
                        part = __shfl_sync(0xffffffffu, scan(part), 31);
                    }
                    if (!by_warp || lane == 0) {
                        sh.at[q] = u + head * all + part;
                        if (q == 0) sh.begin = {i, head, tile, sh.at[0]};
                    }
                    break;
                }
                if (i + 1 < b1) {                     // more than one only where not by_warp
                    int none = 0;
                    u += units_of(i, INT32_MAX, &none) * w.H;
                    i0 += n;
                }
            }
        }
        __syncthreads();
        walk.round = sh.begin;
        walk.start += sh.at[2] - sh.at[0];
        walk.end += sh.at[2] - sh.at[1];
    }
    const int64_t pos = walk.start;
    if (by_warp) {
        const int64_t all = __shfl_sync(0xffffffffu, incl, 31);
        if (lane == 0 && before <= pos && pos < before + all * w.H) {
            sh.seq = b0;
            sh.base = before;
            sh.per_head = all;
        }
    } else {
        int64_t u = before + (incl - mine) * w.H;
        if (u <= pos && pos < u + mine * w.H) {
            for (int i = b0;; ++i) {
                int none = 0;
                const int64_t v = per == 1 ? mine : units_of(i, INT32_MAX, &none);
                if (pos < u + v * w.H) {
                    sh.seq = i;
                    sh.base = u;
                    sh.per_head = v;
                    break;
                }
                u += v * w.H;
            }
        }
    }
    __syncthreads();
    walk.seq = -1;
    walk.here = {w.b.n_seqs, 0, 0, 0};
    walk.stage = 3;
    walk.begun = false;
    walk.kb0 = walk.kb1 = walk.nb = 0;
    if (sh.seq < 0 || walk.start >= walk.end) return;
    walk.stage = 0;
    KvWalk::Item &it = walk.here;
    it.seq = sh.seq;
    it.at = sh.base;
    walk.s.load(w, walk.seq = it.seq);
    it.head = (int)kv_div64(pos - it.at, sh.per_head);
    it.tile = 0;
    it.at += it.head * sh.per_head;
    // the tile, 32 at a time: every warp finds it for itself
    const int tiles = walk.s.tiles(w);
    for (int t0 = 0; tiles > 1; t0 += 32) {
        const int64_t u = t0 + lane < tiles ? kFixedUnits + walk.s.blocks(w, t0 + lane) : 0;
        const int64_t upto = scan(u), all = __shfl_sync(0xffffffffu, upto, 31);
        if (it.at + all <= pos && t0 + 32 < tiles) {
            it.at += all;
            continue;
        }
        const int i = __popc(__ballot_sync(0xffffffffu, it.at + upto <= pos));
        it.at += __shfl_sync(0xffffffffu, upto - u, i);
        it.tile = t0 + i;
        break;
    }
    if (it.at < walk.start) {      // begun by the worker before
        walk.begun = w.split;
        walk.first = it;
        walk.item(w, it);
        walk.advance(w, it);
    }
}

// A slot of the workspace: the sums of one piece, `rows` rows of D unnormalised fp32
// values and their (maximum, sum of weights) after them; a row's maximum is in the
// exponent of two.  Slot 2 c + 1: worker c's piece with its item's last keys (and not the
// first), 2 c: its other piece.
ECHO_DEV float *kv_slot(float *ws, int worker, bool tail, int rows, int D) {
    return ws + (int64_t)(2 * worker + (tail ? 1 : 0)) * rows * (D + 2);
}
// What worker c leaves for the joining kernel, after the slots: the end of its units, and
// the item that it began and those after it went on with, up to unit `upto` (0: none).
struct KvJoin {
    int64_t end, upto;
    int row, packed0, rows, head;      // first row of the sequence; packed rows of the item
};
ECHO_DEV KvJoin *kv_joins(float *ws, const KvWork &w, int D) {
    return reinterpret_cast<KvJoin *>(ws + (int64_t)2 * w.workers * w.slot_rows * (D + 2));
}
// By one thread of each CTA, before the first wait that may give up (the joining kernel runs
// all the same, and takes its addresses from here), and again with walk at its piece with an
// item's last keys.
ECHO_DEV void kv_leave_join(const KvWork &w, const KvWalk &walk, float *ws, int D) {
    if (!w.split) return;
    KvJoin j = {walk.end, 0, 0, 0, 0, 0};
    if (walk.tail()) {
        j.upto = walk.from + kFixedUnits + walk.nb;
        j.row = walk.s.row;
        j.packed0 = walk.tile * w.tile;
        j.rows = min(w.tile, walk.s.packed - j.packed0);
        j.head = walk.head;
    }
    kv_joins(ws, w, D)[blockIdx.x] = j;
}
inline size_t kv_workspace_bytes(int workers, int rows, int D) {
    static_assert(sizeof(KvJoin) % 16 == 0, "");
    return (size_t)workers * (2 * rows * (D + 2) * 4 + sizeof(KvJoin));
}

namespace echo {
// whole_keys: tables that cover no more are not divided, which saves the second launch
inline KvWork kv_work(const KvAttention &a, int tile, int slot_rows, int block_shift, int workers,
                      int whole_keys) {
    const echo_kv_pool &p = *a.pool;
    const int64_t cap = (int64_t)a.batch->max_pages * p.page_tokens;
    KvWork w;
    w.b = kv_batch(*a.batch);
    w.H = p.H;
    w.group = a.Hq / p.H;
    w.causal_block = a.causal_block;
    w.tile = tile;
    w.by_group = KvDiv(w.group);
    w.by_tile = KvDiv(tile);
    w.by_block = KvDiv(a.causal_block > 0 ? a.causal_block : 1);
    w.slot_rows = slot_rows;
    w.cap = (int)(cap < kMostKeys ? cap : kMostKeys);
    w.block_shift = block_shift;
    w.workers = workers;
    w.split = cap > whole_keys;
    return w;
}
void launch_kv_join(const KvAttention &a, const KvWork &w, cudaStream_t st);
}  // namespace echo
