// How the work of one attention call over the paged cache is divided between CTAs
// ("workers"), on the device, since the sequences' lengths are known only there.
//
// Items: (sequence, key/value head, row tile).  The Hq / H query heads that share a
// key/value head are packed with the rows, packed row = row * group + head of the group,
// and a tile is `tile` of them, so that keys and values are read once for all.  An item
// costs kFixed + (its key blocks) units; the items stand in a row, sequence by sequence,
// head by head, tile by tile, and worker c of G takes units [U c / G, U (c + 1) / G).  An
// item that crosses such a boundary is done in pieces: each worker leaves its piece's sums
// in the workspace, and the combining kernel joins them in the order of the keys.  A
// worker has at most one piece that does not begin at its item's beginning (its first) and
// one that begins there but ends early (its last): two slots of workspace each.
#pragma once

#include "kv_pages.cuh"

struct KvWork {
    KvBatch b;
    int H, group, causal_block;
    int tile, slot_rows;   // packed rows of a tile, and rows of a workspace slot
    int cap;               // positions that a table row covers
    int block_shift;       // keys of a block, as a power of two
    int workers, least;    // workers, and the fewest units for one
    int split;             // 0: items are not divided; each goes to the worker of its first unit
};

constexpr int kFixedUnits = 2;   // set-up and end of a piece, in key-block times

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
    ECHO_DEV int tiles(const KvWork &w) const { return (packed + w.tile - 1) / w.tile; }
    // keys that row r sees
    ECHO_DEV int top(const KvWork &w, int r) const {
        if (w.causal_block == 0) return min(len, w.cap);
        const int64_t p = shift + r;
        if (p < 0) return 0;
        const unsigned cb = (unsigned)w.causal_block;
        return (int)min((unsigned)min(len, w.cap), ((unsigned)min(p, (int64_t)INT32_MAX) / cb + 1u) * cb);
    }
    // keys that any row of tile t sees: those of its last row
    ECHO_DEV int keys(const KvWork &w, int t) const {
        const int last = min((t + 1) * w.tile, packed) - 1;
        return top(w, row + last / w.group);
    }
    ECHO_DEV int blocks(const KvWork &w, int t) const {
        return (keys(w, t) + (1 << w.block_shift) - 1) >> w.block_shift;
    }
};

// A worker's walk over its pieces; the same in every thread that keeps one.
struct KvWalk {
    KvSeq s;
    int seq, head, tile;   // of the current piece's item
    int kb0, kb1, nb;      // its key blocks, and the item's
    bool some;             // there has been a piece
    int64_t start, end, at;   // the worker's units, and those passed (the next item's first)
    int64_t total;            // units of all items
    int G;                    // workers that have any
    int nseq, nhead, ntile;   // the next item

    ECHO_DEV int64_t unit_of(int worker) const { return worker < G ? total * worker / G : total; }
    // the first key block of an item (units from ..) that `unit` or a later one pays for
    static ECHO_DEV int block_at(int64_t unit, int64_t from, int nb) {
        return (int)min(max(unit - from - kFixedUnits, (int64_t)0), (int64_t)nb);
    }
    ECHO_DEV bool whole() const { return kb0 == 0 && kb1 == nb; }

    // the next piece that has something to do; false at the end
    ECHO_DEV bool next(const KvWork &w) {
        for (;;) {
            if (nseq >= w.b.n_seqs || at >= end) return false;
            if (nseq != seq) s.load(w, seq = nseq);
            if (s.packed == 0) {
                ++nseq;
                continue;
            }
            head = nhead;
            tile = ntile;
            nb = s.blocks(w, tile);
            const int64_t from = at;
            at += kFixedUnits + nb;
            if (++ntile == s.tiles(w)) {
                ntile = 0;
                if (++nhead == w.H) {
                    nhead = 0;
                    ++nseq;
                }
            }
            if (w.split) {
                if (at <= start) continue;
                kb0 = block_at(start, from, nb);
                kb1 = block_at(end, from, nb);
            } else {
                if (from < start) continue;
                kb0 = 0;
                kb1 = nb;
            }
            if (kb0 < kb1 || (nb == 0 && from >= start)) return some = true;
        }
    }
};

// What the threads of a block find together: the units of all items, and the item that
// holds one unit.
struct KvFound {
    int64_t units[32];
    int64_t base, per_head;
    int seq;
};

// The range of `worker`, and the walk set to the item that holds its first unit.  Called by
// every thread of the block.  Thread t looks
// at sequences [t per, (t + 1) per), or a warp at each where there are no more sequences
// than warps (a long chunk has many tiles).
template <int THREADS>
ECHO_DEV void kv_find(const KvWork &w, int worker, KvFound &sh, KvWalk &walk) {
    constexpr int WARPS = THREADS / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool by_warp = w.b.n_seqs <= WARPS;
    const int per = by_warp ? 1 : (w.b.n_seqs + THREADS - 1) / THREADS;
    const int b0 = by_warp ? warp : (int)threadIdx.x * per;
    auto units_of = [&](int seq, int from, int step) -> int64_t {   // of one head
        KvSeq s;
        s.load(w, seq);
        int64_t u = 0;
        const int tiles = s.tiles(w);
        for (int t = from; t < tiles; t += step) u += kFixedUnits + s.blocks(w, t);
        return u;
    };
    auto scan = [&](int64_t v) -> int64_t {                         // inclusive, over the warp
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t x = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += x;
        }
        return v;
    };
    int64_t mine = 0;
    if (by_warp) {
        if (b0 < w.b.n_seqs) mine = units_of(b0, lane, 32) * w.H;
    } else {
        for (int i = 0; i < per && b0 + i < w.b.n_seqs; ++i) mine += units_of(b0 + i, 0, 1) * w.H;
    }
    const int64_t incl = scan(mine);
    if (lane == 31) sh.units[warp] = incl;
    if (threadIdx.x == 0) sh.seq = -1;
    __syncthreads();
    int64_t before = 0, total = 0;   // of the earlier warps; of all
    for (int i = 0; i < WARPS; ++i) {
        const int64_t v = sh.units[i];
        if (i < warp) before += v;
        total += v;
    }
    const int64_t want = total / w.least + 1;
    walk.total = total;
    walk.G = want < w.workers ? (int)want : w.workers;
    walk.start = walk.unit_of(worker);
    walk.end = walk.unit_of(worker + 1);
    const int64_t pos = walk.start;
    if (by_warp) {
        const int64_t all = __shfl_sync(0xffffffffu, incl, 31);
        if (lane == 0 && before <= pos && pos < before + all) {
            sh.seq = b0;
            sh.base = before;
            sh.per_head = all / w.H;
        }
    } else {
        int64_t u = before + incl - mine;
        if (u <= pos && pos < u + mine) {
            for (int i = 0;; ++i) {
                const int64_t v = units_of(b0 + i, 0, 1);
                if (pos < u + v * w.H) {
                    sh.seq = b0 + i;
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
    walk.nseq = w.b.n_seqs;
    walk.nhead = walk.ntile = 0;
    walk.some = false;
    if (sh.seq < 0 || walk.start >= walk.end) return;
    walk.nseq = sh.seq;
    walk.at = sh.base;
    walk.s.load(w, walk.seq = walk.nseq);
    walk.nhead = (int)((pos - walk.at) / sh.per_head);
    walk.at += walk.nhead * sh.per_head;
    // the tile, 32 at a time: every warp finds it for itself
    const int tiles = walk.s.tiles(w);
    for (int t0 = 0;; t0 += 32) {
        const int64_t u = t0 + lane < tiles ? kFixedUnits + walk.s.blocks(w, t0 + lane) : 0;
        const int64_t upto = scan(u), all = __shfl_sync(0xffffffffu, upto, 31);
        if (walk.at + all <= pos && t0 + 32 < tiles) {
            walk.at += all;
            continue;
        }
        const int i = __popc(__ballot_sync(0xffffffffu, walk.at + upto <= pos));
        walk.at += __shfl_sync(0xffffffffu, upto - u, i);
        walk.ntile = t0 + i;
        return;
    }
}

// A slot of the workspace: the sums of one piece, `rows` rows of D unnormalised fp32
// values and their (maximum, sum of weights) after them; a row's maximum is in the
// exponent of two.  Slot 2 c: worker c's piece that begins inside its item, 2 c + 1: the
// one that begins there and ends early.
ECHO_DEV float *kv_slot(float *ws, int worker, bool first, int rows, int D) {
    return ws + (int64_t)(2 * worker + (first ? 1 : 0)) * rows * (D + 2);
}
// What worker c leaves for the joining kernel, after the slots: its last piece, where that
// begins its item and `more` workers after it go on with it.
struct KvJoin {
    int more, row, packed0, rows, head;   // first row of the sequence; packed rows of the item
};
ECHO_DEV KvJoin *kv_joins(float *ws, const KvWork &w, int D) {
    return reinterpret_cast<KvJoin *>(ws + (int64_t)2 * w.workers * w.slot_rows * (D + 2));
}
// After the last call of walk.next(), by one thread of each CTA.
ECHO_DEV void kv_leave_join(const KvWork &w, const KvWalk &walk, float *ws, int D) {
    if (!w.split) return;
    KvJoin j = {0, 0, 0, 0, 0};
    if (walk.some && walk.kb0 == 0 && walk.kb0 < walk.kb1 && walk.kb1 < walk.nb) {   // the last piece, cut short
        while (walk.unit_of((int)blockIdx.x + 1 + j.more) < walk.at) ++j.more;
        j.row = walk.s.row;
        j.packed0 = walk.tile * w.tile;
        j.rows = min(w.tile, walk.s.packed - j.packed0);
        j.head = walk.head;
    }
    kv_joins(ws, w, D)[blockIdx.x] = j;
}
inline size_t kv_workspace_bytes(int workers, int rows, int D) {
    return (size_t)workers * (2 * rows * (D + 2) * 4 + sizeof(KvJoin));
}

namespace echo {
inline KvWork kv_work(const KvAttention &a, int tile, int slot_rows, int block_shift, int workers) {
    const echo_kv_pool &p = *a.pool;
    const int64_t cap = (int64_t)a.batch->max_pages * p.page_tokens;
    KvWork w;
    w.b = kv_batch(*a.batch);
    w.H = p.H;
    w.group = a.Hq / p.H;
    w.causal_block = a.causal_block;
    w.tile = tile;
    w.slot_rows = slot_rows;
    w.cap = (int)(cap < INT32_MAX ? cap : INT32_MAX);
    w.block_shift = block_shift;
    w.workers = workers;
    w.least = 4;
    w.split = 1;
    return w;
}
void launch_kv_join(const KvAttention &a, const KvWork &w, cudaStream_t st);
}  // namespace echo
