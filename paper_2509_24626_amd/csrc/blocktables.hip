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
// find their sequences in the prefix sum.
#include <algorithm>

#include "internal.hpp"

namespace {

constexpr int kMaxSeqs = 65536;
constexpr int kOneGroupRows = 4096;
constexpr int kFillRows = 1024;     // rows of a workgroup of the fill kernel
constexpr int kReleasePages = 2048;  // table entries of a workgroup of the release copy
constexpr int kOneGroupPages = 16384;

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
__device__ __forceinline__ uint32_t blocks_of(uint32_t n, int shift) { return (n >> shift) + ((n & ((1u << shift) - 1)) ? 1u : 0u); }

struct row_t {
    int slot, pos;
};

// One new token of a sequence: its slot, and its page into the table where it
// is the page's first.  x: the page's number among those the step takes.
__device__ __forceinline__ row_t place_row(uint32_t pos, uint32_t held, uint32_t taken, int n_free, int n_pages, int shift,
                                           const int32_t *__restrict__ free_pages, int32_t *table)
{
    const uint32_t j = pos >> shift;
    int page;
    if (j >= held) {
        const int64_t at = (int64_t)n_free - 1 - taken - (j - held);
        page = at >= 0 ? free_pages[at] : -1;
        if (page < 0 || page >= n_pages) page = -1;
        if ((pos & ((1u << shift) - 1)) == 0) table[j] = page;
    } else {
        page = table[j];
        if (page < 0 || page >= n_pages) page = -1;
    }
    return {page < 0 ? -1 : (page << shift) + (int)(pos & ((1u << shift) - 1)), (int)pos};
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
    const int t = threadIdx.x, lane = t & 63, waves = blockDim.x >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const uint32_t cap = (uint32_t)a.token_cap;
    int n_free = a.n_free[0];
    n_free = n_free < 0 ? 0 : (n_free > a.n_pages ? a.n_pages : n_free);
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
        const bool row_long = !row_bad && after > (uint32_t)a.max_blocks;
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
            if (few) {
                int32_t *table = a.tables + (int64_t)b * a.max_blocks;
                for (uint32_t r = begin; live && r < end; ++r) {
                    row_t x = {-1, -1};
                    if (st == kServed) x = place_row((uint32_t)len + (r - begin), held, taken, n_free, a.n_pages, a.shift, a.free_pages, table);
                    a.slots[r] = x.slot;
                    if (a.positions) a.positions[r] = x.pos;
                }
            } else {
                for (unsigned long long left = __ballot(live && end > begin); left; left &= left - 1) {
                    const int l = __builtin_ctzll(left);
                    const uint32_t len_l = lane_of((uint32_t)len, l), begin_l = lane_of(begin, l), end_l = lane_of(end, l);
                    const uint32_t held_l = lane_of(held, l), taken_l = lane_of(taken, l);
                    const bool served = lane_of((uint32_t)st, l) == kServed;
                    int32_t *table = a.tables + (int64_t)(b0 + wave * 64 + l) * a.max_blocks;
                    for (uint32_t r = begin_l + lane; r < end_l; r += 64) {
                        row_t x = {-1, -1};
                        if (served) x = place_row(len_l + (r - begin_l), held_l, taken_l, n_free, a.n_pages, a.shift, a.free_pages, table);
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

// the last of the sequences [0, n) that begins at or before row r (tok_begin[0] is 0): 64 probes a round
__device__ __forceinline__ int find_seq(const int32_t *__restrict__ tok_begin, int n, uint32_t r, int lane)
{
    int lo = 0;
    for (int span = n; span > 1;) {
        const int step = (span + 63) / 64, b = lo + lane * step;
        const unsigned long long at = __ballot(b < n && (uint32_t)tok_begin[b < n ? b : n - 1] <= r);
        lo += (at ? 63 - __builtin_clzll(at) : 0) * step;
        span = step;
    }
    return lo;
}

// Rows of large batches: what the scan left in tok_begin, taken, status,
// len_out and n_free_out says everything else.
__global__ __launch_bounds__(256) void fill_rows_kernel(const tables_args a)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t cap = (uint32_t)a.token_cap, total = (uint32_t)a.tok_begin[a.B];
    const uint32_t base = (uint32_t)blockIdx.x * kFillRows + wave * 256;
    if (base >= cap) return;
    const int n_free = a.n_free_out[0] + a.taken[a.B];
    int b = 0, last = 0;
    if (base < total) {
        b = find_seq(a.tok_begin, a.B, base, lane);
        last = find_seq(a.tok_begin, a.B, min(base + 255, total - 1), lane);
    }
    const uint32_t r0 = base + lane * 4;
    // this lane's first sequence, in [b, last]
    for (int hi = last; b < hi;) {
        const int mid = (b + hi + 1) >> 1;
        if ((uint32_t)a.tok_begin[mid] <= r0) b = mid;
        else hi = mid - 1;
    }
    i32x4_t slot = {-1, -1, -1, -1}, pos = {-1, -1, -1, -1};
    int of = -1;  // the sequence whose values follow
    uint32_t begin = 0, end = 0, len = 0, held = 0, taken = 0;
    bool served = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t r = r0 + i;
        if (r >= total) break;
        while (b < last && (uint32_t)a.tok_begin[b + 1] <= r) ++b;
        if (b != of) {
            of = b;
            begin = (uint32_t)a.tok_begin[b];
            end = (uint32_t)a.tok_begin[b + 1];
            served = a.status[b] == kServed;
            len = (uint32_t)a.len_out[b] - (end - begin);
            held = blocks_of(len, a.shift);
            taken = (uint32_t)a.taken[b];
        }
        if (served) {
            const row_t x = place_row(len + (r - begin), held, taken, n_free, a.n_pages, a.shift, a.free_pages,
                                      a.tables + (int64_t)b * a.max_blocks);
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
    if (!a.done[b]) return 0;
    const int n = a.len[b];
    return n <= 0 ? 0u : min(blocks_of((uint32_t)n, a.shift), (uint32_t)a.max_blocks);
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

// Entries of one finished sequence's row onto the free list, behind those of
// the finished sequences before it.
__device__ __forceinline__ void push_row(const release_args &a, int b, uint32_t from, uint32_t to, int64_t at)
{
    const int32_t *row = a.tables + (int64_t)b * a.max_blocks;
    for (uint32_t j = from + threadIdx.x; j < to; j += blockDim.x) {
        const int page = row[j];
        if (at + j < a.n_pages) a.free_pages[at + j] = page < 0 || page >= a.n_pages ? -1 : page;
    }
}

__device__ __forceinline__ int clamp_free(const release_args &a)
{
    const int n = a.n_free[0];
    return n < 0 ? 0 : (n > a.n_pages ? a.n_pages : n);
}

// A workgroup copies up to kReleasePages entries of a row; most find a row
// that is not done, or shorter, and leave.  Each sums what the sequences
// before give back itself, so that the copy needs nothing from another launch.
__global__ __launch_bounds__(256) void release_copy_kernel(const release_args a, int chunks)
{
    __shared__ uint32_t s_part[4];
    for (int64_t w = blockIdx.x; w < (int64_t)a.B * chunks; w += gridDim.x) {
        const int b = (int)(w / chunks);
        const uint32_t from = (uint32_t)(w - (int64_t)b * chunks) * kReleasePages, count = gives_back(a, b);
        if (from >= count) continue;
        uint32_t sum = 0;
        for (int i = threadIdx.x; i < b; i += 256) sum = add_sat(sum, gives_back(a, i));
        const uint32_t before = block_sum(sum, s_part);
        push_row(a, b, from, min(count, from + kReleasePages), (int64_t)clamp_free(a) + before);
    }
}

// COPY: the entries too, row after row (small tables)
template <bool COPY>
__global__ __launch_bounds__(1024) void release_kernel(const release_args a)
{
    __shared__ uint32_t s_part[16];
    const int n_free = clamp_free(a);
    uint32_t total = 0;
    if (COPY) {
        const int lane = threadIdx.x & 63;  // a sequence each
        const uint32_t count = lane < a.B ? gives_back(a, lane) : 0u, upto = wave_scan(count);
        for (unsigned long long left = __ballot(count > 0); left; left &= left - 1) {
            const int b = __builtin_ctzll(left);
            const uint32_t n = lane_of(count, b);
            push_row(a, b, 0, n, (int64_t)n_free + (lane_of(upto, b) - n));
        }
        total = lane_of(upto, 63);
        __syncthreads();  // every wave has read the lengths
    } else {
        uint32_t sum = 0;
        for (int b = threadIdx.x; b < a.B; b += blockDim.x) sum = add_sat(sum, gives_back(a, b));
        total = block_sum(sum, s_part);
    }
    for (int b = threadIdx.x; b < a.B; b += blockDim.x) {
        const int n = a.done[b] ? 0 : a.len[b];
        a.len_out[b] = n;
        if (a.nblk_out) a.nblk_out[b] = n < 0 ? 0 : n >> a.shift;
    }
    if (threadIdx.x == 0) a.n_free_out[0] = (int)min((int64_t)n_free + total, (int64_t)a.n_pages);
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
    fill_rows_kernel<<<dim3((token_cap + kFillRows - 1) / kFillRows), dim3(256), 0, s>>>(a);
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
    if ((int64_t)B * max_blocks <= kOneGroupPages && B <= 64) {
        ss::launch(release_kernel<true>, dim3(1), dim3(1024), s, a);
        return ss::check_launch("ss_block_release");
    }
    const int chunks = (int)std::min<int64_t>(((int64_t)max_blocks + kReleasePages - 1) / kReleasePages, kMaxSeqs);
    const int64_t groups = std::min<int64_t>((int64_t)B * chunks, 4096);
    ss::launch(release_copy_kernel, dim3((unsigned)groups), dim3(256), s, a, chunks);
    st = ss::check_launch("ss_block_release");
    if (st) return st;
    release_kernel<false><<<dim3(1), dim3(1024), 0, s>>>(a);
    return ss::check_launch("ss_block_release(lengths)");
}
