// Block tables and slot maps of a shared pool of pages, built on the GPU from
// the requests' lengths (Section 3.1: fixed-size blocks; requests join, grow
// and finish between steps), so that a step needs no host round trip.
//
// Reserving pages is a prefix sum over the sequences: of their new tokens
// (the rows of the step's token tensors) and of the pages that these need.
// Pages are taken from the top of the free list in sequence order, so page x
// of the step is free_pages[n_free - 1 - x], and which sequences are served
// follows from one comparison with the sum of all needs up to there.  The
// sums saturate at 2^32 - 1, far above any pool or batch.
//
// One workgroup scans (a thread per sequence, DPP within a wave, the waves'
// totals through LDS).  Up to kOneGroupRows token rows it also fills the rows
// itself; beyond, a second launch fills 1024 rows a workgroup, whose lanes
// find their sequences in the prefix sums.  Loads that follow one another bound
// it, so what can be loaded early is: the page of a row's open block and the top
// of the free list are on their way while the sums run.  One more token for each
// of 64 sequences takes 2.5 us; a step of 512 sequences, 16 of them prompts of up
// to 16k tokens, 2.8 and 6.2, and the release before it 4.2.
#include <algorithm>

#include "internal.hpp"

namespace {

constexpr int kMaxSeqs = 65536;
// Token rows that the scanning workgroup fills itself.  us, one launch and two, rows
// of 1 token each: 64 3.1, 6.5; 1024 4.3, 8.8; 4096 12.2, 14.8.  A sequence's rows are
// filled by the wave that has it, so a long chunk does not gain: 4 chunks of 250 6.3,
// 6.2; one of 4000 beside 3 tokens 17.7, 6.4, beside 63 37.3, 7.2.
constexpr int kOneGroupRows = 4096;
constexpr int kFillRows = 1024;  // rows of a workgroup of the fill kernel
constexpr int kSearch = 2048;    // entries of tok_begin that it searches in LDS
constexpr int kReleasePages = 2048;  // table entries of a workgroup of the release copy

typedef int i32x4_t __attribute__((ext_vector_type(4), aligned(4)));

enum { kServed = 0, kNoPages = 1, kLongRow = 2, kBadRow = 3 };

__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp0(uint32_t x)  // lanes without a source get 0
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xF, false);
}

// inclusive sum over the wave's lanes, saturating
__device__ __forceinline__ uint32_t wave_scan(uint32_t x)
{
    x = add_sat(x, dpp0<0x111, 0xF>(x));  // row_shr 1, 2, 4, 8
    x = add_sat(x, dpp0<0x112, 0xF>(x));
    x = add_sat(x, dpp0<0x114, 0xF>(x));
    x = add_sat(x, dpp0<0x118, 0xF>(x));
    x = add_sat(x, dpp0<0x142, 0xA>(x));  // lane 15 of rows 0, 2 to rows 1, 3
    x = add_sat(x, dpp0<0x143, 0xC>(x));  // lane 31 to rows 2, 3
    return x;
}

__device__ __forceinline__ uint32_t lane_of(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }

// what blocks of `blk` = 2^shift tokens n tokens take
__device__ __forceinline__ uint32_t blocks_of(uint32_t n, int shift)
{
    return (n >> shift) + ((n & ((1u << shift) - 1)) ? 1u : 0u);
}

struct row_t {
    int slot, pos;
};

// One new token of a sequence: its slot, and its page into the table where it
// is the page's first.  page_of(x): the x-th page from the top of the free
// list; open_page: that of the block in which the tokens held end.
template <class F>
__device__ __forceinline__ row_t place_row(uint32_t pos, uint32_t held, uint32_t taken, int open_page, int n_pages, int shift,
                                           int32_t *table, const F &page_of)
{
    const uint32_t j = pos >> shift, place = pos & ((1u << shift) - 1);
    int page = j >= held ? page_of(taken + (j - held)) : open_page;
    if (page < 0 || page >= n_pages) page = -1;
    if (j >= held && place == 0) table[j] = page;
    return {page < 0 ? -1 : (page << shift) + (int)place, (int)pos};
}

struct tables_args {
    const int32_t *len, *n_new, *n_free;
    int B, shift, max_blocks, n_pages;
    const int32_t *free_pages;
    int32_t *tables, *len_out, *nblk_out, *n_free_out, *tok_begin, *slots, *positions;
    int token_cap;
    int32_t *taken, *status;
};

// FILL: the rows too
template <bool FILL>
__global__ __launch_bounds__(1024) void tables_kernel(const tables_args a)
{
    __shared__ uint32_t s_rows[16], s_need[16], s_good[16];
    __shared__ int s_free[FILL ? 1024 : 1];  // the top of the free list, as far as there are threads
    const int t = threadIdx.x, lane = t & 63, waves = blockDim.x >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const uint32_t cap = (uint32_t)a.token_cap;
    int n_free = a.n_free[0];
    n_free = n_free < 0 ? 0 : (n_free > a.n_pages ? a.n_pages : n_free);
    if (FILL) s_free[t] = t < n_free ? a.free_pages[n_free - 1 - t] : -1;
    uint32_t rows0 = 0, need0 = 0, good0 = 0;  // sums of the chunks before; pages taken so far
    for (int b0 = 0; b0 < a.B; b0 += blockDim.x) {
        const int b = b0 + t;
        const bool live = b < a.B;
        int len = 0, n = 0;
        if (live) {
            len = a.len[b];
            n = a.n_new[b];
        }
        const bool bad = len < 0 || n < 0;
        int open_page = -1;  // of the block that the row's tokens so far end in
        if (FILL && !bad && live && (len >> a.shift) < a.max_blocks)
            open_page = a.tables[(int64_t)b * a.max_blocks + (len >> a.shift)];
        const uint32_t nn = n < 0 ? 0u : (uint32_t)n;
        const uint32_t rows = wave_scan(nn);
        if (lane == 63) s_rows[wave] = rows;
        __syncthreads();
        // a sequence whose rows pass token_cap takes no pages, so the rows come first
        const uint32_t rt = lane < waves ? s_rows[lane] : 0u;
        const uint32_t rscan = wave_scan(rt);
        const uint32_t rows_end = add_sat(rows0, add_sat(wave ? lane_of(rscan, wave - 1) : 0u, rows));
        const uint32_t held = bad ? 0u : blocks_of((uint32_t)len, a.shift);
        const uint32_t after = bad ? 0u : blocks_of((uint32_t)len + nn, a.shift);
        const bool row_bad = bad || (nn > 0 && rows_end > cap);
        const bool row_long = !row_bad && (after > (uint32_t)a.max_blocks || (uint32_t)len + nn > 0x7FFFFFFFu);
        const uint32_t need = row_bad || row_long ? 0u : after - held;
        const uint32_t upto_w = wave_scan(need);
        if (lane == 63) s_need[wave] = upto_w;
        __syncthreads();
        const uint32_t nt = lane < waves ? s_need[lane] : 0u;
        const uint32_t nscan = wave_scan(nt);
        const uint32_t upto = add_sat(need0, add_sat(wave ? lane_of(nscan, wave - 1) : 0u, upto_w));
        // taken before b: the sum of the needs before it, or, once a sequence
        // has gone without, the largest sum that the pool could meet
        const bool meets = upto <= (uint32_t)n_free;
        const unsigned long long met = __ballot(meets);
        const uint32_t good_w = met ? lane_of(upto, 63 - __builtin_clzll(met)) : 0u;  // upto does not fall from lane to lane
        if (lane == 0) s_good[wave] = good_w;
        __syncthreads();
        uint32_t good = good0;
        for (int w = 0; w < waves; ++w) good = max(good, s_good[w]);
        const bool hit = need > 0 && !meets;
        const int st = row_bad ? kBadRow : row_long ? kLongRow : hit ? kNoPages : kServed;
        const uint32_t before = upto - need;  // sums that saturate are above n_free either way
        const uint32_t taken = before <= (uint32_t)n_free ? before : good;
        const uint32_t begin = min(rows_end - nn, cap), end = min(rows_end, cap);
        if (live) {
            const uint32_t nlen = st == kServed ? (uint32_t)len + nn : (uint32_t)len;
            a.len_out[b] = (int)nlen;
            if (a.nblk_out) a.nblk_out[b] = len < 0 ? 0 : (int)(nlen >> a.shift);
            a.tok_begin[b] = (int)begin;
            a.taken[b] = (int)taken;
            a.status[b] = st;
        }
        if (FILL) {
            // a lane's own rows one by one where every sequence has few (a decode
            // step), else the wave's sequences in turn, 64 rows at once
            const bool few = !__any(live && nn > 4);
            auto page_of = [&](uint32_t x) {
                return x < blockDim.x ? s_free[x] : x < (uint32_t)n_free ? a.free_pages[n_free - 1 - x] : -1;
            };
            if (few) {
                int32_t *table = a.tables + (int64_t)b * a.max_blocks;
                for (uint32_t r = begin; live && r < end; ++r) {
                    row_t x = {-1, -1};
                    if (st == kServed)
                        x = place_row((uint32_t)len + (r - begin), held, taken, open_page, a.n_pages, a.shift, table, page_of);
                    a.slots[r] = x.slot;
                    if (a.positions) a.positions[r] = x.pos;
                }
            } else {
                for (unsigned long long left = __ballot(live && end > begin); left; left &= left - 1) {
                    const int l = __builtin_ctzll(left);
                    const uint32_t len_l = lane_of((uint32_t)len, l), begin_l = lane_of(begin, l), end_l = lane_of(end, l);
                    const uint32_t held_l = lane_of(held, l), taken_l = lane_of(taken, l);
                    const int open_l = (int)lane_of((uint32_t)open_page, l);
                    const bool served = lane_of((uint32_t)st, l) == kServed;
                    int32_t *table = a.tables + (int64_t)(b0 + wave * 64 + l) * a.max_blocks;
                    for (uint32_t r = begin_l + lane; r < end_l; r += 64) {
                        row_t x = {-1, -1};
                        if (served)
                            x = place_row(len_l + (r - begin_l), held_l, taken_l, open_l, a.n_pages, a.shift, table, page_of);
                        a.slots[r] = x.slot;
                        if (a.positions) a.positions[r] = x.pos;
                    }
                }
            }
        }
        rows0 = add_sat(rows0, lane_of(rscan, 63));
        need0 = add_sat(need0, lane_of(nscan, 63));
        good0 = good;
    }
    const uint32_t total = min(rows0, cap);
    if (t == 0) {
        a.tok_begin[a.B] = (int)total;
        a.taken[a.B] = (int)good0;
        a.n_free_out[0] = n_free - (int)good0;
    }
    if (FILL)
        for (uint32_t r = total + t; r < cap; r += blockDim.x) {
            a.slots[r] = -1;
            if (a.positions) a.positions[r] = -1;
        }
}

struct seq_t {
    uint32_t len, held, taken;  // tokens and pages before the step, pages taken before the sequence
    bool served;
};

// Rows of large batches: what the scan left in tok_begin, taken, status,
// len_out and n_free_out says everything else.  The row's sequence is found in
// a copy of tok_begin in LDS (of every `step`-th entry where there are more
// than fit, the rest from memory), so that three loads follow one another:
// tok_begin, the sequence, the page.  Four rows that cross an end go on sequence by
// sequence, so idle ones between two live ones cost a step each (8190 of them 570 us,
// 19 without).
__global__ __launch_bounds__(256) void fill_rows_kernel(const tables_args a)
{
    __shared__ uint32_t s_begin[kSearch];
    const uint32_t cap = (uint32_t)a.token_cap, total = (uint32_t)a.tok_begin[a.B];
    const int n_free = a.n_free_out[0] + a.taken[a.B];
    const int step = (a.B + kSearch - 1) / kSearch, n = (a.B + step - 1) / step;
    for (int i = threadIdx.x; i < n; i += 256) s_begin[i] = (uint32_t)a.tok_begin[i * step];
    __syncthreads();
    const uint32_t r0 = (uint32_t)blockIdx.x * kFillRows + threadIdx.x * 4;
    // the last sequence that begins at or before a row (tok_begin[0] is 0): for
    // the wave's first row and its last together, 64 probes at once; only
    // where they differ does a lane look for its own
    const int lane = threadIdx.x & 63;
    const uint32_t w0 = (uint32_t)blockIdx.x * kFillRows + (threadIdx.x - lane) * 4;
    auto last_of = [](unsigned long long at) { return at ? 63 - __builtin_clzll(at) : 0; };
    constexpr int kCoarse = kSearch / 64;
    const int i0 = lane * kCoarse;
    const uint32_t x = i0 < n ? s_begin[i0] : ~0u;
    const int lo0 = last_of(__ballot(x <= w0)) * kCoarse, hi0 = last_of(__ballot(x <= w0 + 255)) * kCoarse;
    const uint32_t y = lane < kCoarse && lo0 + lane < n ? s_begin[lo0 + lane] : ~0u;
    const uint32_t z = lane < kCoarse && hi0 + lane < n ? s_begin[hi0 + lane] : ~0u;
    int b = lo0 + last_of(__ballot(y <= w0));
    for (int hi = hi0 + last_of(__ballot(z <= w0 + 255)); b < hi;) {
        const int mid = (b + hi + 1) >> 1;
        if (s_begin[mid] <= r0) b = mid;
        else hi = mid - 1;
    }
    b *= step;
    for (int hi = min(b + step, a.B) - 1; b < hi;) {
        const int mid = (b + hi + 1) >> 1;
        if ((uint32_t)a.tok_begin[mid] <= r0) b = mid;
        else hi = mid - 1;
    }
    if (r0 >= cap) return;
    auto page_of = [&](uint32_t i) { return i < (uint32_t)n_free ? a.free_pages[n_free - 1 - i] : -1; };
    i32x4_t slot = {-1, -1, -1, -1}, pos = {-1, -1, -1, -1};
    uint32_t begin = 0, end = 0;
    seq_t q = {};
    int32_t *table = nullptr;
    auto enter = [&] {  // sequence b
        begin = (uint32_t)a.tok_begin[b];
        end = (uint32_t)a.tok_begin[b + 1];
        const uint32_t len = (uint32_t)a.len_out[b];
        const uint32_t taken = (uint32_t)a.taken[b];
        q.served = a.status[b] == kServed;
        q.len = len - (end - begin);
        q.held = blocks_of(q.len, a.shift);
        q.taken = taken;
        table = a.tables + (int64_t)b * a.max_blocks;
    };
    enter();
    if (r0 + 4 <= end && r0 >= begin) {
        // four rows of one sequence, as most are: they lie in one block or two
        if (q.served) {
            const uint32_t p0 = q.len + (r0 - begin), mask = (1u << a.shift) - 1;
            const uint32_t j0 = p0 >> a.shift, j1 = (p0 + 3) >> a.shift;
            int first = j0 >= q.held ? page_of(q.taken + (j0 - q.held)) : table[j0];
            int second = j1 >= q.held ? page_of(q.taken + (j1 - q.held)) : table[j1];
            if (first < 0 || first >= a.n_pages) first = -1;
            if (second < 0 || second >= a.n_pages) second = -1;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t p = p0 + i, j = p >> a.shift;
                const int page = j == j0 ? first : second;
                slot[i] = page < 0 ? -1 : (page << a.shift) + (int)(p & mask);
                pos[i] = (int)p;
                if ((p & mask) == 0 && j >= q.held) table[j] = page;
            }
        }
    } else {
        for (int i = 0; i < 4; ++i) {
            const uint32_t r = r0 + i;
            if (r >= total) break;
            while (r >= end) {
                ++b;
                enter();
            }
            if (!q.served) continue;
            const uint32_t at = q.len + (r - begin);
            const int open_page = (at >> a.shift) < q.held ? table[at >> a.shift] : -1;
            const row_t x = place_row(at, q.held, q.taken, open_page, a.n_pages, a.shift, table, page_of);
            slot[i] = x.slot;
            pos[i] = x.pos;
        }
    }
    if (r0 + 4 <= cap) {
        *reinterpret_cast<i32x4_t *>(a.slots + r0) = slot;
        if (a.positions) *reinterpret_cast<i32x4_t *>(a.positions + r0) = pos;
    } else {
        for (int i = 0; i < 4 && r0 + i < cap; ++i) {
            a.slots[r0 + i] = slot[i];
            if (a.positions) a.positions[r0 + i] = pos[i];
        }
    }
}

struct release_args {
    const int32_t *len, *done, *n_free;
    int B, shift, max_blocks, n_pages;
    const int32_t *tables;
    int32_t *free_pages, *len_out, *nblk_out, *n_free_out;
};

// pages that sequence b gives back
__device__ __forceinline__ uint32_t gives_back(const release_args &a, int b)
{
    const int done = a.done[b], n = a.len[b];  // neither load waits for the other
    return done && n > 0 ? min(blocks_of((uint32_t)n, a.shift), (uint32_t)a.max_blocks) : 0u;
}

__device__ __forceinline__ uint32_t block_sum(uint32_t x, uint32_t *s_part)
{
    x = lane_of(wave_scan(x), 63);
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = x;
    __syncthreads();
    uint32_t sum = 0;
    for (unsigned w = 0; w < blockDim.x >> 6; ++w) sum = add_sat(sum, s_part[w]);
    __syncthreads();
    return sum;
}

__device__ __forceinline__ uint32_t sum_before(const release_args &a, int n, uint32_t *s_part)
{
    uint32_t sum = 0;
    for (int i = threadIdx.x; i < n; i += blockDim.x) sum = add_sat(sum, gives_back(a, i));
    return block_sum(sum, s_part);
}

__device__ __forceinline__ void put_lengths(const release_args &a, int from, int stride)
{
    for (int b = from; b < a.B; b += stride) {
        const int n = a.done[b] ? 0 : a.len[b];
        a.len_out[b] = n;
        if (a.nblk_out) a.nblk_out[b] = n < 0 ? 0 : n >> a.shift;
    }
}

// A workgroup copies up to kReleasePages entries of a row behind those of the
// finished rows before it; most find a row that is not done, or shorter, and
// go on.  Each sums what the rows before give back itself, so that the copy
// needs nothing from another launch.  LENGTHS: the lengths and the count too,
// where they are written apart from what is read.
template <bool LENGTHS>
__global__ __launch_bounds__(256) void release_kernel(const release_args a, int chunks)
{
    __shared__ uint32_t s_part[4];
    int n_free = a.n_free[0];
    n_free = n_free < 0 ? 0 : (n_free > a.n_pages ? a.n_pages : n_free);
    for (int64_t w = blockIdx.x; w < (int64_t)a.B * chunks; w += gridDim.x) {
        const int b = (int)(w / chunks);
        const uint32_t from = (uint32_t)(w - (int64_t)b * chunks) * kReleasePages, count = gives_back(a, b);
        if (from >= count) continue;
        const int64_t at = (int64_t)n_free + sum_before(a, b, s_part);
        const int32_t *row = a.tables + (int64_t)b * a.max_blocks;
        const uint32_t to = min(count, from + kReleasePages);
        for (uint32_t j = from + threadIdx.x; j < to; j += 256) {
            const int page = row[j];
            if (at + j < a.n_pages) a.free_pages[at + j] = page < 0 || page >= a.n_pages ? -1 : page;
        }
    }
    if (LENGTHS) {
        put_lengths(a, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
        if (blockIdx.x == gridDim.x - 1) {
            const int64_t all = (int64_t)n_free + sum_before(a, a.B, s_part);
            if (threadIdx.x == 0) a.n_free_out[0] = (int)min(all, (int64_t)a.n_pages);
        }
    }
}

// the lengths and the count where they are updated in place
__global__ __launch_bounds__(1024) void release_lengths_kernel(const release_args a)
{
    __shared__ uint32_t s_part[16];
    int n_free = a.n_free[0];
    n_free = n_free < 0 ? 0 : (n_free > a.n_pages ? a.n_pages : n_free);
    const int64_t all = (int64_t)n_free + sum_before(a, a.B, s_part);
    put_lengths(a, threadIdx.x, blockDim.x);
    if (threadIdx.x == 0) a.n_free_out[0] = (int)min(all, (int64_t)a.n_pages);
}

int shift_of(int blk) { return blk == 8 ? 3 : blk == 16 ? 4 : 5; }

ss_status check_pool(const char *who, int B, int blk, int max_blocks, int n_pages)
{
    SS_CHECK_ARG(B >= 0 && max_blocks > 0 && n_pages >= 0, "%s: bad shape B=%d max_blocks=%d n_pages=%d", who, B, max_blocks,
                 n_pages);
    SS_CHECK_SUPPORTED(ss::supported_blk(blk), "%s: blk=%d (8, 16 or 32)", who, blk);
    SS_CHECK_SUPPORTED(B <= kMaxSeqs, "%s: B=%d > %d", who, B, kMaxSeqs);
    SS_CHECK_SUPPORTED((int64_t)n_pages * blk <= 0x7FFFFFFF, "%s: the slots of %d pages pass 32 bits", who, n_pages);
    return SS_OK;
}

}  // namespace

extern "C" ss_status ss_block_tables(const int32_t *len, const int32_t *n_new, const int32_t *n_free, int B, int blk,
                                     int max_blocks, int n_pages, const int32_t *free_pages, int32_t *tables,
                                     int32_t *len_out, int32_t *nblk_out, int32_t *n_free_out, int32_t *tok_begin,
                                     int32_t *slots, int32_t *positions, int token_cap, int32_t *taken, int32_t *status,
                                     void *stream)
{
    ss_status st = check_pool("ss_block_tables", B, blk, max_blocks, n_pages);
    if (st) return st;
    SS_CHECK_ARG(token_cap >= 0, "ss_block_tables: token_cap=%d", token_cap);
    if (B == 0) return SS_OK;
    SS_CHECK_ARG(len && n_new && n_free && tables && len_out && n_free_out && tok_begin && taken && status &&
                     (free_pages || n_pages == 0) && (slots || token_cap == 0),
                 "ss_block_tables: null pointer");
    const tables_args a = {len, n_new, n_free, B, shift_of(blk), max_blocks, n_pages, free_pages, tables, len_out,
                           nblk_out, n_free_out, tok_begin, slots, positions, token_cap, taken, status};
    hipStream_t s = ss::as_stream(stream);
    const bool one = token_cap <= kOneGroupRows;
    const dim3 block(std::min(1024, (B + 63) / 64 * 64));
    ss::launch(one ? tables_kernel<true> : tables_kernel<false>, dim3(1), block, s, a);
    st = ss::check_launch("ss_block_tables");
    if (st != SS_OK || one) return st;
    fill_rows_kernel<<<dim3((token_cap - 1) / kFillRows + 1), dim3(256), 0, s>>>(a);
    return ss::check_launch("ss_block_tables(rows)");
}

extern "C" ss_status ss_block_release(const int32_t *len, const int32_t *done, const int32_t *n_free, int B, int blk,
                                      int max_blocks, int n_pages, const int32_t *tables, int32_t *free_pages,
                                      int32_t *len_out, int32_t *nblk_out, int32_t *n_free_out, void *stream)
{
    ss_status st = check_pool("ss_block_release", B, blk, max_blocks, n_pages);
    if (st) return st;
    if (B == 0) return SS_OK;
    SS_CHECK_ARG(len && done && n_free && tables && len_out && n_free_out && (free_pages || n_pages == 0),
                 "ss_block_release: null pointer");
    const release_args a = {len, done, n_free, B, shift_of(blk), max_blocks, n_pages, tables, free_pages, len_out,
                            nblk_out, n_free_out};
    hipStream_t s = ss::as_stream(stream);
    const int chunks = (max_blocks - 1) / kReleasePages + 1;
    const int64_t groups = std::min<int64_t>((int64_t)B * chunks, 4096);
    const bool apart = len_out != len && n_free_out != n_free;
    ss::launch(apart ? release_kernel<true> : release_kernel<false>, dim3((unsigned)groups), dim3(256), s, a, chunks);
    st = ss::check_launch("ss_block_release");
    if (st != SS_OK || apart) return st;
    release_lengths_kernel<<<dim3(1), dim3(1024), 0, s>>>(a);
    return ss::check_launch("ss_block_release(lengths)");
}
