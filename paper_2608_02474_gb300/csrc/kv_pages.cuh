// The paged key/value cache (echo_kv_pool, echo_kv_batch of echocache.h) as the
// kernels see it: where a row's keys and values stand.
#pragma once

#include "common.cuh"
#include "internal.h"

// a pool by value: pages [n_pages, 2, H, 1 << shift, d], scale [n_pages, 2, H, 1 << shift]; for
// 4-bit codes pages [.., d / 2] bytes, scale bf16 [.., 1 << shift, d / 32]
struct KvPool {
    uint8_t *pages;
    void *scale;
    int n_pages, shift, H;
};

// What pages hold, as a constant of the kernels: an echo_cache_kind.
constexpr int kBf16 = ECHO_CACHE_BF16, kInt8 = ECHO_CACHE_INT8, kInt4 = ECHO_CACHE_INT4;
constexpr int kv_bytes(int form, int values) {
    return form == kInt4 ? values / 2 : form == kInt8 ? values : 2 * values;
}

struct KvBatch {
    const int32_t *table, *len, *row0;
    int n_seqs, max_pages, n_rows;
};

// The sequence that row r belongs to and the row's position in it; seq -1 where there is
// none.  It is the last b with row0[b] <= r if row0[b + 1] lies beyond r.  The whole warp
// searches for one row, 32 entries at a time: two dependent loads for up to 1024 sequences,
// where a bisection takes ten.
struct KvRow {
    int seq;
    int64_t p;
};
ECHO_DEV KvRow kv_find_row(const KvBatch &b, int r) {
    const int lane = threadIdx.x & 31;
    int lo = 0, n = b.n_seqs;
    while (n > 1) {
        const int step = (n + 31) >> 5, i = lane * step;
        const int below = __popc(__ballot_sync(0xffffffffu, i < n && b.row0[lo + i] <= r));
        if (below == 0) return {-1, 0};
        const int skip = (below - 1) * step;
        lo += skip;
        n = min(step, n - skip);
    }
    const int first = b.row0[lo], end = b.row0[lo + 1], len = b.len[lo];   // at once
    return {first <= r && r < end ? lo : -1, (int64_t)len - end + r};
}

// Place of position p of a sequence in the pool, as page * (1 << shift) + slot; -1 where the
// sequence's table does not lead to a page of the pool, which sets the device flag.
ECHO_DEV int64_t kv_place(const KvPool &pool, const KvBatch &b, int seq, int64_t p, int *err) {
    const int64_t i = p >> pool.shift;
    const int page = i < b.max_pages ? b.table[(int64_t)seq * b.max_pages + i] : -1;
    if ((unsigned)page >= (unsigned)pool.n_pages) {
        echo_flag_error(err, ECHO_ERR_PAGE);
        return -1;
    }
    return ((int64_t)page << pool.shift) + (p & ((1 << pool.shift) - 1));
}

// Four int8 codes as bf16 pairs of code / 64, exactly.  With the sign bit flipped a byte is
// u = code + 128; a 16-bit half with u in its low byte and 0 above is the bf16 number
// u 2^-133 (below 128 a subnormal one, and bf16 fma takes those), and
// u 2^-133 2^127 - 2 = (u - 128) / 64 needs no more than 7 bits.  The selectors pick the two
// bytes of a pair (4: a zero byte).
constexpr float kCodeUnit = 64.f;   // what the scales are multiplied by in return
ECHO_DEV uint32_t kv_flip(uint32_t w) { return w ^ 0x80808080u; }
ECHO_DEV uint32_t kv_codes2(uint32_t flipped, uint32_t sel) {
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;"
        : "=r"(r)
        : "r"(__byte_perm(flipped, 0u, sel)), "r"(0x7F007F00u), "r"(0xC000C000u));   // 2^127, -2
    return r;
}

// Four-bit codes of two columns, nibble I of w's halves, as a bf16 pair of code / 64, exactly: as
// for int8, the nibbles stand alone in the halves as numbers of 2^-133 (the higher one of a byte as 16
// times that, bit 7 being the first of the exponents'), and a fused multiply-add makes (n - 8) / 64 of
// them.  A shift serves two nibbles: the integer pipe, of half the rate, is the one that fills up.
constexpr float kNibbleUnit = 64.f;   // what scores and sums are multiplied by in return
template <int I>
ECHO_DEV uint32_t kv_nibbles2(uint32_t w) {
    const uint32_t x = (I < 2 ? w : w >> 8) & (I % 2 ? 0x00F000F0u : 0x000F000Fu);
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;"
        : "=r"(r)
        : "r"(x), "r"(I % 2 ? 0x7D007D00u : 0x7F007F00u), "r"(0xBE00BE00u));   // 2^123 or 2^127, -1 / 8
    return r;
}
// times the scales of two columns or keys: code s / 64, exact for s of 5 significant bits
ECHO_DEV uint32_t bf16x2_mul(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <int I>
ECHO_DEV uint32_t kv_nibbles2(uint32_t w, uint32_t s2) { return bf16x2_mul(kv_nibbles2<I>(w), s2); }
// the halves of a pair of bf16 that are not finite: all ones there
ECHO_DEV uint32_t kv_not_finite2(uint32_t v) {
    return ((v & 0x7F80u) == 0x7F80u ? 0xffffu : 0u) | ((v & 0x7F800000u) == 0x7F800000u ? 0xffff0000u : 0u);
}

namespace echo {
// argument checks of the entry points; ECHO_OK with *empty set: there is nothing to do
echo_status kv_check(const echo_kv_pool *pool, const echo_kv_batch *batch, bool *empty);
inline int kv_shift(int page_tokens) {
    int s = 0;
    while ((1 << s) < page_tokens) ++s;
    return s;
}
inline KvPool kv_pool(const echo_kv_pool &p) {
    return {static_cast<uint8_t *>(p.pages), p.scale, p.n_pages, kv_shift(p.page_tokens), p.H};
}
inline KvBatch kv_batch(const echo_kv_batch &b) {
    return {b.table, b.len, b.row0, b.n_seqs, b.max_pages, b.n_rows};
}
}  // namespace echo
