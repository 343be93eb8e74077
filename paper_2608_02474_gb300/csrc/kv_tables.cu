// Page tables, first rows and slot maps of a step, made on the device from how many new
// tokens each sequence has, and sequences shortened again.
//
// Both are sums over the sequences (pages that those before a sequence take, rows that they
// have) and then independent entries.  One launch: each CTA of a cluster computes the sums of
// all sequences for itself (8192 of them are 32 KB an array, from the L2), and the cluster
// shares out the entries (those of many rows are left to a second launch); a cluster barrier between
// the two parts keeps the tables as they were until everybody has read them.  The bytes of a row's place, position and
// sequence are 16, so what a call takes is its latency: launch, reading lengths, the sums' barriers,
// and the chain from an entry's search to its page.  Long tables are an exception: the used entries of the step's own
// table are copied, by 8 SMs at most (512 sequences of 32760 tokens in pages of 16, extended and shortened again:
// 29.9 us for 8.4 MB, 1.2 us at the rate of a copy; 1000 tokens in pages of 64 each, and 500 more: 15.2).
#include "common.cuh"
#include "internal.h"

namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kMostSeqs = 8192, kMostSlots = 1 << 18;
constexpr int kRowsHere = 8192;                       // rows whose maps the first launch makes
constexpr int kMostTokens = INT32_MAX / 128 * 128;   // of a sequence, as the attention takes them

struct Tables {
    int32_t *table, *len, *free_pages, *n_free;
    int n_pages, shift, n_slots, max_pages;
};
struct Step {
    const int32_t *slots, *rows;
    int32_t *table, *len, *row0, *pos, *seq;
    int64_t *place;
    int n_seqs, n_rows;
    bool rows_here;              // the row maps, too
};

// exclusive sums of two numbers over the CTA's threads, and their totals; `part` [2][kWarps]
struct Sums {
    int64_t a, b;
};
ECHO_DEV Sums scan(Sums v, int64_t (*part)[kWarps], Sums &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Sums in = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t a = __shfl_up_sync(0xffffffffu, in.a, o), b = __shfl_up_sync(0xffffffffu, in.b, o);
        if (lane >= o) in.a += a, in.b += b;
    }
    if (lane == 31) part[0][warp] = in.a, part[1][warp] = in.b;
    __syncthreads();
    int64_t a = part[0][lane], b = part[1][lane];     // kWarps = 32
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(0xffffffffu, a, o), y = __shfl_up_sync(0xffffffffu, b, o);
        if (lane >= o) a += x, b += y;
    }
    total = {__shfl_sync(0xffffffffu, a, 31), __shfl_sync(0xffffffffu, b, 31)};
    const int before = max(warp - 1, 0);
    const int64_t pa = __shfl_sync(0xffffffffu, a, before), pb = __shfl_sync(0xffffffffu, b, before);
    __syncthreads();
    return {in.a - v.a + (warp ? pa : 0), in.b - v.b + (warp ? pb : 0)};
}

// EXTEND or shorten.  Shared memory: the sequences' first rows (shorten: tokens given up), slots, lengths, the
// pages that they have before (shorten: keep after) and the pages moved before theirs; a bit
// for each slot that is named.
template <bool EXTEND>
__global__ void __launch_bounds__(kThreads)
kv_tables_kernel(const Tables t, const Step s, int *err) {
    extern __shared__ int32_t smem[];
    __shared__ int64_t part[2][kWarps];
    __shared__ int bad;
    const int n = s.n_seqs, tid = threadIdx.x;
    int32_t *row0 = smem, *slot = row0 + n + 1, *len = slot + n, *have = len + n, *before = have + n;
    uint32_t *named = reinterpret_cast<uint32_t *>(before + n);
    for (int i = tid; i < (t.n_slots + 31) / 32; i += kThreads) named[i] = 0u;
    if (tid == 0) bad = 0;
    pdl_enter();
    const int n_free = *t.n_free;
    const int64_t most = min((int64_t)t.max_pages << t.shift, (int64_t)kMostTokens);
    const int page = 1 << t.shift;
    __syncthreads();
    Sums carry = {0, 0};
    bool wrong = n_free < 0 || n_free > t.n_pages;
    for (int base = 0; base < n; base += kThreads) {
        const int i = base + tid;
        Sums v = {0, 0};
        int id = -1, l = 0, h = 0;
        if (i < n) {
            id = s.slots ? s.slots[i] : i;
            int64_t r = s.rows[i];
            if ((unsigned)id < (unsigned)t.n_slots) {
                wrong |= (atomicOr(&named[id >> 5], 1u << (id & 31)) >> (id & 31)) & 1u;
                l = t.len[id];
            } else {
                id = -1;
            }
            if (!EXTEND) r = min(r, (int64_t)l);
            if (id < 0 || r < 0 || l < 0 || l > most || (EXTEND && (l + r > most || r > s.n_rows))) {
                wrong = true;
                r = 0;
                l = max(l, 0);
            }
            const int now = (int)(((int64_t)l + page - 1) >> t.shift);
            if (EXTEND) {
                h = now;
                v = {r, ((l + r + page - 1) >> t.shift) - now};
            } else {
                h = (int)((l - r + page - 1) >> t.shift);
                v = {r, now - h};
            }
        }
        Sums total;
        const Sums at = scan(v, part, total);
        if (i < n) {
            slot[i] = id;
            len[i] = l;
            have[i] = h;
            before[i] = (int)min(carry.b + at.b, (int64_t)INT32_MAX);   // past 2^31 the call is refused
            // shorten: the sequence's own number, since the sum may pass 31 bits
            row0[i] = EXTEND ? (int)min(carry.a + at.a, (int64_t)INT32_MAX) : (int)v.a;
            if (EXTEND && i == n - 1) row0[n] = (int)min(carry.a + at.a + v.a, (int64_t)INT32_MAX);
        }
        carry.a += total.a;
        carry.b += total.b;
    }
    if (n == 0 && tid == 0) row0[0] = 0;
    if (EXTEND) wrong |= carry.a > s.n_rows || carry.b > n_free;
    else wrong |= n_free + carry.b > t.n_pages;
    if (wrong) bad = 1;
    // everybody has read the tables, and every thread knows whether the call can be served
    const int ranks = (int)cluster_nctarank(), rank = (int)cluster_ctarank();
    if (ranks > 1) cluster_sync_all();
    __syncthreads();
    const bool ok = bad == 0;
    const int moved = (int)carry.b;
    if (rank == 0) {
        if (!ok && tid == 0) echo_flag_error(err, ECHO_ERR_PAGE);
        if (ok && tid == 0) *t.n_free = EXTEND ? n_free - moved : n_free + moved;
        for (int i = tid; i < n; i += kThreads) {
            const int rows = EXTEND ? row0[i + 1] - row0[i] : row0[i];
            const int to = !ok ? len[i] : EXTEND ? len[i] + rows : len[i] - rows;
            if (ok) t.len[slot[i]] = to;
            if (EXTEND) {
                s.len[i] = to;
                s.row0[i + 1] = ok ? row0[i + 1] : 0;
            }
        }
        if (EXTEND && tid == 0) s.row0[0] = 0;
    }
    if (EXTEND) {
        // rows: the last b with row0[b] <= r, over the copy in shared memory; many rows are left
        // to kv_rows_kernel
        const int live = ok ? row0[n] : 0;
        for (int64_t r0 = (int64_t)rank * kThreads + tid; s.rows_here && r0 < s.n_rows; r0 += (int64_t)ranks * kThreads) {
            const int r = (int)r0;
            int64_t place = -1;
            int p = -1, b = -1;
            if (r < live) {
                int lo = 0, width = n;                // the answer is in [lo, lo + width)
                while (width > 1) {
                    const int half = width >> 1;
                    if (row0[lo + half] <= r) lo += half, width -= half;
                    else width = half;
                }
                b = lo;
                p = len[b] + (r - row0[b]);
                const int j = p >> t.shift;
                const int id = j < have[b] ? t.table[(int64_t)slot[b] * t.max_pages + j]
                                           : t.free_pages[n_free - 1 - (before[b] + j - have[b])];
                place = ((int64_t)id << t.shift) + (p & (page - 1));
            }
            if (s.place) s.place[r] = place;
            if (s.pos) s.pos[r] = p;
            if (s.seq) s.seq[r] = b;
        }
    }
    if (!ok) return;
    // pages: as many threads to a sequence as there are, a warp at least
    const int threads = ranks * kThreads;
    int width = 32;
    while (width < threads && 2 * width * n <= threads) width *= 2;
    const int me = rank * kThreads + tid, lane = me & (width - 1);
    for (int b = me / width; b < n; b += threads / width) {
        int32_t *own = t.table + (int64_t)slot[b] * t.max_pages;
        if (EXTEND) {
            const int rows = row0[b + 1] - row0[b];
            const int want = (int)(((int64_t)len[b] + rows + page - 1) >> t.shift);
            int32_t *out = s.table ? s.table + (int64_t)b * t.max_pages : nullptr;
#pragma unroll 4
            for (int j = (out ? 0 : have[b]) + lane; j < want; j += width) {
                const bool fresh = j >= have[b];
                const int id = fresh ? t.free_pages[n_free - 1 - (before[b] + j - have[b])] : own[j];
                if (fresh) own[j] = id;
                if (out) out[j] = id;
            }
        } else {
            const int had = (int)(((int64_t)len[b] + page - 1) >> t.shift);
            for (int j = have[b] + lane; j < had; j += width)
                t.free_pages[n_free + moved - 1 - (before[b] + j - have[b])] = own[j];
        }
    }
}

// The maps of many rows, four neighbouring ones to a thread, from the tables as they are now: a launch of
// its own, since a cluster is 8 SMs (240000 rows of five sequences extended and shortened again: in
// the cluster's own launch 24.5 us, so 11.8).
template <bool WIDE>
__global__ void __launch_bounds__(256) kv_rows_kernel(const Tables t, const Step s) {
    pdl_enter();
    const int live = s.row0[s.n_seqs];
    const int64_t first = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x);
    if (first >= s.n_rows) return;
    int b = 0, from = 0, to = 0, len = 0, slot = 0, page_at = -1, page = 0;
    int64_t place[4];
    int pos[4], seq[4];
    if (first < live) {
        int width = s.n_seqs;                         // the answer is in [b, b + width)
        while (width > 1) {
            const int half = width >> 1;
            if (s.row0[b + half] <= first) b += half, width -= half;
            else width = half;
        }
    }
    auto load = [&]() {
        from = s.row0[b];
        to = s.row0[b + 1];
        len = s.len[b];
        slot = s.slots ? s.slots[b] : b;
        page_at = -1;
    };
    if (first < live) load();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int64_t r = first + k;
        place[k] = pos[k] = seq[k] = -1;
        if (r >= live) continue;
        while (r >= to) {                             // row0 ends above every live row
            ++b;
            load();
        }
        seq[k] = b;
        pos[k] = len - to + (int)r;
        const int j = pos[k] >> t.shift;
        if (j != page_at) page = t.table[(int64_t)slot * t.max_pages + (page_at = j)];
        place[k] = ((int64_t)page << t.shift) + (pos[k] & ((1 << t.shift) - 1));
    }
    if (WIDE && first + 3 < s.n_rows) {
        if (s.place) {
            reinterpret_cast<longlong2 *>(s.place + first)[0] = make_longlong2(place[0], place[1]);
            reinterpret_cast<longlong2 *>(s.place + first)[1] = make_longlong2(place[2], place[3]);
        }
        if (s.pos) *reinterpret_cast<int4 *>(s.pos + first) = make_int4(pos[0], pos[1], pos[2], pos[3]);
        if (s.seq) *reinterpret_cast<int4 *>(s.seq + first) = make_int4(seq[0], seq[1], seq[2], seq[3]);
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (first + k >= s.n_rows) continue;
        if (s.place) s.place[first + k] = place[k];
        if (s.pos) s.pos[first + k] = pos[k];
        if (s.seq) s.seq[first + k] = seq[k];
    }
}

__global__ void __launch_bounds__(256) kv_tables_reset_kernel(const Tables t) {
    pdl_enter();
    const int at = blockIdx.x * 256 + threadIdx.x, step = gridDim.x * 256;
    for (int64_t i = at; i < t.n_slots; i += step) t.len[i] = 0;
    for (int64_t i = at; i < t.n_pages; i += step) t.free_pages[i] = t.n_pages - 1 - (int)i;
    if (at == 0) *t.n_free = t.n_pages;
}

bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

echo_status check(const echo_kv_tables *t) {
    if (!t) return ECHO_ERR_INVALID_ARG;
    if (t->n_pages < 1 || t->n_slots < 1 || t->n_slots > kMostSlots || t->max_pages < 1) return ECHO_ERR_SHAPE;
    if ((int64_t)t->n_slots * t->max_pages > INT32_MAX) return ECHO_ERR_SHAPE;
    if (t->page_tokens != 16 && t->page_tokens != 32 && t->page_tokens != 64 && t->page_tokens != 128)
        return ECHO_ERR_SHAPE;
    for (const void *p : {(const void *)t->table, (const void *)t->len, (const void *)t->free_pages,
                          (const void *)t->n_free})
        if (!p || !aligned4(p)) return ECHO_ERR_INVALID_ARG;
    return ECHO_OK;
}

Tables tables(const echo_kv_tables &t) {
    int shift = 0;
    while ((1 << shift) < t.page_tokens) ++shift;
    return {t.table, t.len, t.free_pages, t.n_free, t.n_pages, shift, t.n_slots, t.max_pages};
}

template <bool EXTEND>
echo_status launch(const echo_kv_tables &t, const Step &s, cudaStream_t st) {
    // an entry or four a thread; 8 CTAs: the largest cluster that every GPU has
    const int64_t entries = (s.rows_here ? (int64_t)s.n_rows : 0) + (int64_t)s.n_seqs * t.max_pages;
    unsigned ranks = 1;
    while (ranks < 8 && ranks * 4 * (int64_t)kThreads < entries) ranks *= 2;
    const size_t smem = 4 * (5 * (size_t)s.n_seqs + 1 + ((size_t)t.n_slots + 31) / 32);
    static int attr_done[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev >= 0 && dev < 64 && !attr_done[dev]) {
        constexpr int kMost = 4 * (5 * kMostSeqs + 1 + kMostSlots / 32);
        cudaFuncSetAttribute(kv_tables_kernel<EXTEND>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
        attr_done[dev] = 1;
    }
    echo::LaunchScope ls(ECHO_K_KV_TABLES, s.n_rows, s.n_seqs, EXTEND ? 0 : 1, st);
    echo::launch_chained_cluster(ranks, kv_tables_kernel<EXTEND>, dim3(ranks), dim3(kThreads), smem, st,
                                 tables(t), s, echo::device_error_ptr());
    return echo::last_launch_status();
}

}  // namespace

extern "C" echo_status echo_kv_tables_reset(const echo_kv_tables *t, echo_stream_t stream) {
    const echo_status ok = check(t);
    if (ok != ECHO_OK) return ok;
    if (!echo::device_supported()) return ECHO_ERR_UNSUPPORTED;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const int most = t->n_pages > t->n_slots ? t->n_pages : t->n_slots;
    const int grid = most / 256 + 1 < 304 ? most / 256 + 1 : 304;
    echo::LaunchScope ls(ECHO_K_KV_TABLES, t->n_pages, t->n_slots, 2, st);
    echo::launch_chained(kv_tables_reset_kernel, dim3(grid), dim3(256), 0, st, tables(*t));
    return echo::last_launch_status();
}

extern "C" echo_status echo_kv_extend(const echo_kv_tables *t, const int32_t *slots, const int32_t *rows,
                                      int32_t n_seqs, int32_t n_rows, int32_t *table, int32_t *len,
                                      int32_t *row0, int64_t *place, int32_t *pos, int32_t *seq,
                                      echo_stream_t stream) {
    const echo_status ok = check(t);
    if (ok != ECHO_OK) return ok;
    if (n_seqs < 0 || n_seqs > kMostSeqs || n_rows < 0) return ECHO_ERR_SHAPE;
    if (!row0 || (n_seqs > 0 && (!rows || !len))) return ECHO_ERR_INVALID_ARG;
    for (const void *p : {(const void *)slots, (const void *)rows, (const void *)table, (const void *)len,
                          (const void *)row0, (const void *)pos, (const void *)seq})
        if (!aligned4(p)) return ECHO_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(place) & 7u) return ECHO_ERR_INVALID_ARG;
    if (!echo::device_supported()) return ECHO_ERR_UNSUPPORTED;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool maps = place || pos || seq, apart = maps && n_rows > kRowsHere && n_seqs > 0;
    const Step s = {slots, rows, table, len, row0, pos, seq, place, n_seqs, n_rows, maps && !apart};
    const echo_status done = launch<true>(*t, s, st);
    if (done != ECHO_OK || !apart) return done;
    const int grid = (int)(((int64_t)n_rows + 1023) / 1024);
    const bool wide = echo::aligned16(place) && echo::aligned16(pos) && echo::aligned16(seq);
    echo::LaunchScope ls(ECHO_K_KV_TABLES, n_rows, n_seqs, 0, st);
    echo::launch_chained(wide ? kv_rows_kernel<true> : kv_rows_kernel<false>, dim3(grid), dim3(256), 0, st, tables(*t), s);
    return echo::last_launch_status();
}

extern "C" echo_status echo_kv_shorten(const echo_kv_tables *t, const int32_t *slots, const int32_t *rows,
                                       int32_t n_seqs, echo_stream_t stream) {
    const echo_status ok = check(t);
    if (ok != ECHO_OK) return ok;
    if (n_seqs < 0 || n_seqs > kMostSeqs) return ECHO_ERR_SHAPE;
    if (n_seqs == 0) return ECHO_OK;
    if (!rows || !aligned4(rows) || !aligned4(slots)) return ECHO_ERR_INVALID_ARG;
    if (!echo::device_supported()) return ECHO_ERR_UNSUPPORTED;
    return launch<false>(*t, {slots, rows, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, n_seqs, 0, false},
                         reinterpret_cast<cudaStream_t>(stream));
}
