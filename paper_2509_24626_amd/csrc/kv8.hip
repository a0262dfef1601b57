// The KV cache held in 8 bits: new tokens into block records with a scale for
// each block and head (Section 3.1's fixed-size blocks of one head), and
// records back as bf16 rows.
//
// A block is quantised once, when its last token arrives, from its bf16
// tokens: the ones of earlier calls from the sequence's open record (the
// layout of ss_append_kv), the others from the new rows.  The tokens of a
// block that does not fill stay bf16 in the open record, so no value is
// rounded twice.  With m the largest magnitude of the K (or V) tile, at least
// 2^-100, and Q the largest code (448 of e4m3, 127):
//     scale = m / Q,   code = rne(x * (Q / m)),   value = code * scale
// each step one rounded fp32 operation, so that the result does not depend on
// the shape of the launch.
//
// A team of 64 lanes (32 for blocks of 8) writes the K or the V tile of one
// block of one head, and a workgroup is a wave of K teams beside one of V teams:
// neither tile needs the other, and a wave's chain of dependent loads and its
// arithmetic set the time of all but the largest calls (both tiles to a team: 8
// chunks of 256 tokens, blocks of 32, mean keys 12.4 us, now 8.1; one token for
// each of 64 sequences 4.8 and 4.4; 128k tokens 153 both ways).  16 lanes read
// 256 B of a token, so the tile is in the team's registers with a load per 4
// tokens in flight each, and the codes leave as 16-byte stores.  Teams of
// neighbouring heads are neighbours, so that together they read whole tokens.
// Reading back is split the same way, and a team takes at most 16 tokens (64k
// tokens, 8 heads, blocks of 16 77.5 us with both tiles to a team, now 71; 7
// sequences of up to 5000, 2 heads, blocks of 32 8.6 with a block to a team, now
// 7.0).  Larger workgroups gain nothing, and single waves take 73 us.
// HBM bounds it: 512 B in and 256 B (and 8 per token for the trailer at 16
// tokens a block) out per token and head, and the block's metadata: 128k tokens
// of 8 heads with cuboids 154 us, 5.5 TB/s, read and write together (a large
// copy moves 4.9); reading 64k tokens back 71 us, 5.7 TB/s.
#include <algorithm>

#include "bf16_keys.hpp"
#include "kv8.hpp"

namespace {

constexpr int D = ss::kHeadDim;

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b)  // unsigned halves
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, a),
                                                                  __builtin_bit_cast(u16x2_t, b)));
}

template <int CTRL>
__device__ __forceinline__ uint32_t max2_dpp(uint32_t x)
{
    return max2(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, false));
}

// largest halves over the team, in every lane
template <int TEAM>
__device__ __forceinline__ uint32_t team_max2(uint32_t x)
{
    x = max2_dpp<0xB1>(x);   // lane ^ 1
    x = max2_dpp<0x4E>(x);   // lane ^ 2
    x = max2_dpp<0x141>(x);  // mirrored in 8 lanes
    x = max2_dpp<0x140>(x);  // mirrored in 16 lanes
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max2(r[0], r[1]);
    if (TEAM == 64) {
        const auto h = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        x = max2(h[0], h[1]);
    }
    return x;
}

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
// channel e of 8 in a lane's 16 bytes
__device__ __forceinline__ float channel(const u32x4_t &w, int e) { return e & 1 ? bf16_hi(w[e >> 1]) : bf16_lo(w[e >> 1]); }

// four values, scaled, as codes in the bytes of a register
template <int FMT>
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inv)
{
    // each product is rounded by itself: a fused multiply-add would round a code differently
#pragma clang fp contract(off)
    if constexpr (FMT == SS_KV8_E4M3) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
    } else {
        // 1.5 * 2^23 added: the sum's low bits are the integer, rounded to nearest even
        constexpr float kMagic = 12582912.f;
        const float x = a * inv, y = b * inv, z = c * inv, u = d * inv;
        const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(y + kMagic), __float_as_uint(x + kMagic), 0x0C0C0400);
        const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(u + kMagic), __float_as_uint(z + kMagic), 0x04000C0C);
        return lo | hi;
    }
}

// a tile's scale and its inverse from the bits of its largest magnitude
template <int FMT>
struct tile_scale {
    float scale, inv;
    uint32_t keep;  // 0 where the tile holds an infinity or a NaN: codes 0, scale NaN
    __device__ explicit tile_scale(uint32_t bits)
    {
        constexpr float kQ = FMT == SS_KV8_E4M3 ? 448.f : 127.f;
        const float m = fmaxf(__uint_as_float(bits << 16), 0x1p-100f);
        const bool ok = bits < 0x7F80u;
        keep = ok ? ~0u : 0u;
        inv = kQ / m;
        scale = ok ? m / kQ : __uint_as_float(0x7FC00000u);
    }
};

__device__ __forceinline__ u32x4_t load16(const uint8_t *p) { return *reinterpret_cast<const u32x4_t *>(p); }
__device__ __forceinline__ u32x4_t load16_stream(const uint8_t *p)
{
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p));
}
// Stores are streamed too: writing 64k tokens in blocks of 8 took 90.8 us with
// the default policy, 74.9 so; reading 64k tokens 85.0 and 81.4.  It needs
// whole lines (K codes stored 32 bytes at a time: 97.3).
__device__ __forceinline__ void store16(uint8_t *p, u32x4_t x)
{
    __builtin_nontemporal_store(x, reinterpret_cast<u32x4_t *>(p));
}

constexpr int kThreads = 128;  // of a workgroup

struct write_args {
    const uint8_t *k, *v;
    int64_t tok_stride, head_stride;
    const int32_t *tok_begin, *slots, *positions;
    int B, Hkv, token_cap;
    uint8_t *kv;
    const int64_t *region_off;
    int32_t slot_limit;
    uint8_t *open, *meta;
    int nblk_max;
    int64_t teams;
};

constexpr int kNoMeta = -1;

template <int BLK, int FMT, int META>
__global__ __launch_bounds__(kThreads) void write_kernel(const write_args a)
{
    constexpr int TEAM = BLK == 8 ? 32 : 64;
    constexpr int SUB = BLK == 32 ? 2 : 1, T = BLK / SUB;
    constexpr int NR = 4 * SUB;  // rows of a lane
    constexpr int REC = ss::kv8_record(BLK), OPEN = 2 * BLK * D * 2;
    const int lane = threadIdx.x & 63, tl = lane % TEAM, x = lane & 15, L = tl >> 4;
    const bool is_v = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t team = (blockIdx.x * 64 + lane) / TEAM, item = team / (uint32_t)a.Hkv;
    const int g = (int)(team - item * (uint32_t)a.Hkv);
    const int b = ss::find_item<BLK, TEAM>(a.tok_begin, a.B, item, lane);
    const int64_t u = (int64_t)b * a.Hkv + g;
    const int tb = a.tok_begin[b], n = min(a.tok_begin[b + 1], a.token_cap) - tb;
    int64_t region = a.region_off[u];
    const int64_t m64 = (int64_t)item - (b + (int64_t)(tb / BLK));
    if (team >= a.teams || tb < 0 || n <= 0 || m64 < 0 || m64 > n / BLK) return;  // the whole team
    const int s0 = a.slots[tb];
    if (s0 < 0) return;  // a sequence that found no pages
    const int m = (int)m64, p0 = s0 % BLK;
    const int full = (p0 + n) / BLK;  // blocks that fill
    if (m >= max(full, 1)) return;
    uint8_t *open = a.open + u * OPEN;
    const uint8_t *src = (is_v ? a.v : a.k) + g * a.head_stride + x * 16;

    if (full > 0) {
        u32x4_t R[NR];
        const int i0 = tb + m * BLK - p0;  // the token of the block's row 0
        // where the block goes, beside its rows and not after them
        int last = a.slots[i0 + BLK - 1], pos = META == kNoMeta ? 0 : a.positions[i0 + BLK - 1];
        const int held = m == 0 ? p0 : 0;  // rows of the open record
        const uint8_t *src0 = src + (int64_t)(i0 + 4 * L) * a.tok_stride;
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            const int row = (r >> 2) * 16 + 4 * L + (r & 3);
            const int64_t at = ((r >> 2) * 16 + (r & 3)) * a.tok_stride;
            const uint8_t *p = src0 + at;
            if (row < held) p = open + row * (D * 2) + x * 16;  // V is replaced below
            R[r] = load16_stream(p);
        }
        asm volatile("" : "+v"(last), "+v"(pos), "+v"(region));
        if (is_v && held > 0) {
            const uint8_t *ov = open + BLK * D * 2;
#pragma unroll
            for (int s = 0; s < SUB; ++s) {
                u32x2_t w[8];  // 4 tokens of each channel
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    w[e] = *reinterpret_cast<const u32x2_t *>(ov + ((8 * x + e) * BLK + s * 16 + 4 * L) * 2);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (s * 16 + 4 * L + i < held) {
#pragma unroll
                        for (int h = 0; h < 4; ++h) {
                            const uint32_t lo = w[2 * h][i >> 1], hi = w[2 * h + 1][i >> 1];
                            R[4 * s + i][h] = i & 1 ? (lo >> 16) | (hi & 0xFFFF0000u) : (lo & 0xFFFFu) | (hi << 16);
                        }
                    }
            }
        }
        uint32_t m2 = 0;  // largest magnitudes of both halves
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int h = 0; h < 4; ++h) m2 = max2(m2, R[r][h] & 0x7FFF7FFFu);
        m2 = team_max2<TEAM>(m2);
        const tile_scale<FMT> sc(max(m2 & 0xFFFFu, m2 >> 16));

        const int page = last / BLK;
        if (last >= 0 && page < a.slot_limit && last % BLK == BLK - 1) {
            uint8_t *rec = a.kv + region + (int64_t)page * REC;
#pragma unroll
            for (int s = 0; s < SUB; ++s) {
                uint8_t *kt = rec + s * T * D, *vt = rec + BLK * D + s * T * D;
                if (!is_v) {
                    // rows 4L + 2j and 4L + 2j + 1: the even lane of a pair takes
                    // both lanes' channels of the first, the odd one of the second
                    const bool odd = x & 1;
                    u32x4_t o[2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        uint32_t c[2][2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const u32x4_t w = R[4 * s + 2 * j + i];
                            c[i][0] = codes4<FMT>(channel(w, 0), channel(w, 1), channel(w, 2), channel(w, 3), sc.inv) & sc.keep;
                            c[i][1] = codes4<FMT>(channel(w, 4), channel(w, 5), channel(w, 6), channel(w, 7), sc.inv) & sc.keep;
                        }
                        const uint32_t r0 = ss::pair_swap(odd ? c[0][0] : c[1][0]), r1 = ss::pair_swap(odd ? c[0][1] : c[1][1]);
                        o[j] = odd ? u32x4_t{r0, r1, c[1][0], c[1][1]} : u32x4_t{c[0][0], c[0][1], r0, r1};
                    }
                    // the team's halves exchange, so that a store has 8 (a team of
                    // 32: 4) consecutive tokens of every 16 channels, whole lines
#pragma unroll
                    for (int h = 0; h < 4; ++h) {
                        const auto y = TEAM == 64 ? __builtin_amdgcn_permlane32_swap(o[0][h], o[1][h], false, false)
                                                  : __builtin_amdgcn_permlane16_swap(o[0][h], o[1][h], false, false);
                        o[0][h] = y[0];
                        o[1][h] = y[1];
                    }
                    constexpr int HALF = TEAM / 32;  // lane rows of half a team
                    uint8_t *kl = kt + (x >> 1) * (T * 16) + (4 * (L % HALF) + 2 * (L / HALF) + (odd ? 1 : 0)) * 16;
                    asm("" : "+v"(o[0]), "+v"(o[1]));  // else the two stores lose their policy in compilation
                    store16(kl, o[0]);
                    store16(kl + HALF * 64, o[1]);
                } else {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        u32x4_t o;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            o[e] = codes4<FMT>(channel(R[4 * s], 4 * h + e), channel(R[4 * s + 1], 4 * h + e),
                                               channel(R[4 * s + 2], 4 * h + e), channel(R[4 * s + 3], 4 * h + e), sc.inv) & sc.keep;
                        store16(vt + h * (T * 64) + L * 256 + x * 16, o);
                    }
                }
            }
            uint8_t *trailer = rec + 2 * BLK * D;  // the zeros come with the V scale
            if (tl == 0) reinterpret_cast<float *>(trailer)[is_v] = sc.scale;
            if (is_v && tl == 0) *reinterpret_cast<u32x2_t *>(trailer + 8) = u32x2_t{0, 0};
            if (is_v && tl > 0 && tl < ss::kKv8Trailer / 16) store16(trailer + tl * 16, u32x4_t{0, 0, 0, 0});
        }
        if (META != kNoMeta && !is_v) {
            const int jb = pos / BLK;
            const bool live = pos >= 0 && jb < a.nblk_max;
            if (META == SS_META_CUBOID) {
                u32x4_t o;
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    uint32_t lo = ss::key2(R[0][h]), nhi = ~lo;
#pragma unroll
                    for (int r = 1; r < NR; ++r) {
                        const uint32_t key = ss::key2(R[r][h]);
                        lo = ss::min2(lo, key);
                        nhi = ss::min2(nhi, ~key);
                    }
                    // lane rows 0, 1 (row 0 of a team of 32) end with the minima, the others with the maxima
                    uint32_t y;
                    if (TEAM == 32) {
                        y = ss::min_rows(lo, nhi);
                    } else {
                        y = ss::min_halves(lo, nhi);
                        y = ss::min_rows(y, y);
                    }
                    o[h] = ss::key2(2 * L >= TEAM / 16 ? ~y : y);
                }
                const int hi = 2 * L >= TEAM / 16 ? 1 : 0;
                if (live && L == hi * (TEAM / 32))
                    store16(a.meta + (u * a.nblk_max + jb) * (int64_t)(4 * D) + hi * (2 * D) + x * 16, o);
            } else {
                // the team's lanes exchange, so that each sums all rows of its own 4 (a
                // team of 64: 2) channels
                constexpr int W = 64 / TEAM;  // words of two channels
                uint32_t t[2 * NR][2], w[BLK][W];
#pragma unroll
                for (int r = 0; r < NR; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const auto y = TEAM == 64 ? __builtin_amdgcn_permlane32_swap(R[r][h], R[r][2 + h], false, false)
                                                  : __builtin_amdgcn_permlane16_swap(R[r][h], R[r][2 + h], false, false);
                        t[2 * r][h] = y[0];
                        t[2 * r + 1][h] = y[1];
                    }
#pragma unroll
                for (int r = 0; r < 2 * NR; ++r) {
                    if constexpr (TEAM == 64) {
                        const auto y = __builtin_amdgcn_permlane16_swap(t[r][0], t[r][1], false, false);
                        w[2 * r][0] = y[0];
                        w[2 * r + 1][0] = y[1];
                    } else {
                        w[r][0] = t[r][0];
                        w[r][1] = t[r][1];
                    }
                }
                uint8_t *mean = a.meta + (u * a.nblk_max + jb) * (int64_t)(2 * D) + x * 16 + L * (W * 4);
#pragma unroll
                for (int h = 0; h < W; ++h) {
                    double lo = 0.0, hi = 0.0;
#pragma unroll
                    for (int r = 0; r < BLK; ++r) {
                        lo += (double)bf16_lo(w[r][h]);
                        hi += (double)bf16_hi(w[r][h]);
                    }
                    if (live) reinterpret_cast<uint32_t *>(mean)[h] = ss::pack_bf16_rne_f64(lo * (1.0 / BLK), hi * (1.0 / BLK));
                }
            }
        }
    }

    // the rows of the block that stays open, by the team that read the open record
    const int rest = p0 + n - full * BLK;
    if (m == 0 && rest > 0) {
        __threadfence_block();  // its reads are done
        const int from = full ? 0 : p0, i0 = tb + full * BLK - p0;
        uint16_t *ov = reinterpret_cast<uint16_t *>(open + BLK * D * 2);
        for (int row = from + L; row < rest; row += TEAM / 16) {
            const u32x4_t w = load16(src + (int64_t)(i0 + row) * a.tok_stride);
            if (is_v) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    ov[(8 * x + e) * BLK + row] = (uint16_t)(e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xFFFFu);
            } else {
                store16(open + row * (D * 2) + x * 16, w);
            }
        }
    }
}

struct read_args {
    const uint8_t *kv;
    const int64_t *region_off;
    const int32_t *tables;
    int max_blocks;
    int32_t slot_limit;
    const uint8_t *open;
    const int32_t *len, *row_begin;
    int B, Hkv, rows;
    uint8_t *k, *v;
    int64_t row_stride, head_stride;
    int64_t teams;
};

// two codes (bytes 2*HI, 2*HI + 1 of w), scaled and rounded once to bf16
template <int FMT, bool HI>
__device__ __forceinline__ f32x2_t values2(uint32_t w)
{
    if constexpr (FMT == SS_KV8_E4M3) {
        return __builtin_amdgcn_cvt_pk_f32_fp8((int)w, HI);
    } else {
        return f32x2_t{(float)(int8_t)(w >> (HI ? 16 : 0)), (float)(int8_t)(w >> (HI ? 24 : 8))};
    }
}

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{a, b}, bf16x2_t));
}

// four codes of neighbouring channels -> two registers of bf16
template <int FMT>
__device__ __forceinline__ u32x2_t row4(uint32_t w, float s)
{
    const f32x2_t a = values2<FMT, false>(w), b = values2<FMT, true>(w);
    return u32x2_t{pack2(a.x * s, a.y * s), pack2(b.x * s, b.y * s)};
}

template <int BLK, int FMT>
__global__ __launch_bounds__(kThreads) void read_kernel(const read_args a)
{
    constexpr int TEAM = BLK == 8 ? 32 : 64;
    constexpr int SUB = BLK == 32 ? 2 : 1, T = BLK / SUB;  // a team reads a subtile
    constexpr int REC = ss::kv8_record(BLK), OPEN = 2 * BLK * D * 2;
    const int lane = threadIdx.x & 63, tl = lane % TEAM, x = lane & 15, L = tl >> 4;
    const bool is_v = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t team = (blockIdx.x * 64 + lane) / TEAM, item = team / (uint32_t)a.Hkv;
    const int g = (int)(team - item * (uint32_t)a.Hkv);
    const int b = ss::find_item<T, TEAM>(a.row_begin, a.B, item, lane);
    const int64_t u = (int64_t)b * a.Hkv + g;
    const int rb = a.row_begin[b], len = a.len[b];
    int64_t region = a.region_off[u];
    const int n = min(min(a.row_begin[b + 1], a.rows) - rb, len);
    const int64_t i64 = (int64_t)item - (b + (int64_t)(rb / T));
    if (team >= a.teams || rb < 0 || n <= 0 || i64 < 0 || i64 > (n - 1) / T) return;
    const int i0 = (int)i64 * T, here = min(n - i0, T);  // rows from i0 on
    const int j = i0 / BLK, s = SUB == 1 ? 0 : i0 % BLK / T;
    const int64_t out0 = (int64_t)(rb + i0) * a.row_stride + g * a.head_stride + x * 16;
    uint8_t *out = (is_v ? a.v : a.k) + out0;
    if (j >= len / BLK) {  // the open record's rows
        const uint8_t *open = a.open + u * OPEN;
        const uint16_t *ov = reinterpret_cast<const uint16_t *>(open + BLK * D * 2);
        for (int r = L; r < here; r += TEAM / 16) {
            const int p = s * T + r;
            u32x4_t w;
            if (is_v) {
#pragma unroll
                for (int h = 0; h < 4; ++h) w[h] = ov[(8 * x + 2 * h) * BLK + p] | (uint32_t)ov[(8 * x + 2 * h + 1) * BLK + p] << 16;
            } else {
                w = load16(open + p * (D * 2) + x * 16);
            }
            store16(out + r * a.row_stride, w);
        }
        return;
    }
    int page = j;
    if (a.tables) page = j < a.max_blocks ? a.tables[(int64_t)b * a.max_blocks + j] : -1;
    asm volatile("" : "+v"(region));  // loaded beside the table's entry, not after it
    const bool ok = page >= 0 && page < a.slot_limit;
    const uint8_t *rec = a.kv + region + (int64_t)(ok ? page : 0) * REC;
    u32x4_t c[2] = {};
    float scale = 0.f;
    if (ok) {
        scale = reinterpret_cast<const float *>(rec + 2 * BLK * D)[is_v];
        const uint8_t *kt = rec + s * T * D + (x >> 1) * (T * 16) + (4 * L + (x & 1)) * 16;
        const uint8_t *vt = rec + BLK * D + s * T * D + L * 256 + x * 16;
#pragma unroll
        for (int i = 0; i < 2; ++i) c[i] = load16(is_v ? vt + i * (T * 64) : kt + i * 32);
    }
    u32x4_t o[4];  // rows 4L .. 4L + 3
    if (is_v) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {  // channels 8x + e, 8x + e + 1
            const uint32_t w0 = c[e >> 2][e & 3], w1 = c[e >> 2][(e & 3) + 1];
            const f32x2_t a0 = values2<FMT, false>(w0), a1 = values2<FMT, true>(w0);
            const f32x2_t b0 = values2<FMT, false>(w1), b1 = values2<FMT, true>(w1);
            o[0][e >> 1] = pack2(a0.x * scale, b0.x * scale);
            o[1][e >> 1] = pack2(a0.y * scale, b0.y * scale);
            o[2][e >> 1] = pack2(a1.x * scale, b1.x * scale);
            o[3][e >> 1] = pack2(a1.y * scale, b1.y * scale);
        }
    } else {
        // a lane holds 16 channels of one of two rows; the pair exchanges so that each has 8 of both
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const u32x4_t w = c[i];
            const bool odd = x & 1;
            const uint32_t r0 = ss::pair_swap(odd ? w[0] : w[2]), r1 = ss::pair_swap(odd ? w[1] : w[3]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool mine = odd == (h == 1);
                const u32x2_t lo = row4<FMT>(mine ? (odd ? w[2] : w[0]) : r0, scale);
                const u32x2_t hi = row4<FMT>(mine ? (odd ? w[3] : w[1]) : r1, scale);
                o[2 * i + h] = u32x4_t{lo.x, lo.y, hi.x, hi.y};
            }
        }
    }
    out += 4 * L * a.row_stride;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (4 * L + i < here) store16(out + i * a.row_stride, o[i]);
}

template <int FMT, int META>
auto write_of(int blk)
{
    return blk == 8 ? write_kernel<8, FMT, META> : blk == 16 ? write_kernel<16, FMT, META> : write_kernel<32, FMT, META>;
}

template <int FMT>
auto read_of(int blk)
{
    return blk == 8 ? read_kernel<8, FMT> : blk == 16 ? read_kernel<16, FMT> : read_kernel<32, FMT>;
}

ss_status check_kv8(const char *who, int B, int Hkv, int blk, int d, int fmt, int32_t slot_limit)
{
    SS_CHECK_ARG(B >= 0 && Hkv > 0 && slot_limit >= 0, "%s: bad shape B=%d Hkv=%d slot_limit=%d", who, B, Hkv, slot_limit);
    SS_CHECK_ARG(fmt == SS_KV8_E4M3 || fmt == SS_KV8_INT8, "%s: format %d", who, fmt);
    SS_CHECK_SUPPORTED(d == D, "%s: d=%d (only 128)", who, d);
    SS_CHECK_SUPPORTED(ss::supported_blk(blk), "%s: blk=%d (8, 16 or 32)", who, blk);
    return SS_OK;
}

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

// workgroups; a team is 64 lanes of each of its waves, 32 for blocks of 8
int64_t groups_of(int64_t teams, int blk) { return blk == 8 ? (teams + 1) / 2 : teams; }

}  // namespace

extern "C" size_t ss_kv8_record_bytes(int blk, int d)
{
    return d == D && ss::supported_blk(blk) ? (size_t)ss::kv8_record(blk) : 0;
}

extern "C" ss_status ss_write_kv8(const void *k, const void *v, int64_t tok_stride, int64_t head_stride,
                                  const int32_t *tok_begin, const int32_t *slots, const int32_t *positions, int B, int Hkv,
                                  int blk, int d, int token_cap, int fmt, void *kv_base, const int64_t *region_off,
                                  int32_t slot_limit, void *open_blocks, void *meta, int meta_kind, int nblk_max,
                                  void *stream)
{
    ss_status st = check_kv8("ss_write_kv8", B, Hkv, blk, d, fmt, slot_limit);
    if (st) return st;
    SS_CHECK_ARG(token_cap >= 0, "ss_write_kv8: token_cap=%d", token_cap);
    SS_CHECK_ARG(tok_stride >= 0 && head_stride >= 0 && tok_stride % 16 == 0 && head_stride % 16 == 0,
                 "ss_write_kv8: strides %lld, %lld are no multiples of 16", (long long)tok_stride, (long long)head_stride);
    if (meta) {
        SS_CHECK_ARG(meta_kind == SS_META_CUBOID || meta_kind == SS_META_MEAN, "ss_write_kv8: metadata kind %d", meta_kind);
        SS_CHECK_ARG(nblk_max >= 0 && (positions || token_cap == 0), "ss_write_kv8: metadata needs positions and nblk_max >= 0");
    }
    if (B == 0 || token_cap == 0) return SS_OK;
    SS_CHECK_ARG(k && v && tok_begin && slots && kv_base && region_off && open_blocks, "ss_write_kv8: null pointer");
    SS_CHECK_ARG(aligned16(k) && aligned16(v) && aligned16(kv_base) && aligned16(open_blocks) && aligned16(meta),
                 "ss_write_kv8: buffers must be 16-byte aligned");
    const int64_t teams = ((int64_t)B + token_cap / blk) * Hkv, groups = groups_of(teams, blk);
    SS_CHECK_SUPPORTED(groups <= 0x7FFFFFFF / kThreads, "ss_write_kv8: %lld block records pass the launch",
                       (long long)teams);
    const write_args a = {static_cast<const uint8_t *>(k), static_cast<const uint8_t *>(v), tok_stride, head_stride,
                          tok_begin, slots, positions, B, Hkv, token_cap, static_cast<uint8_t *>(kv_base), region_off,
                          slot_limit, static_cast<uint8_t *>(open_blocks), static_cast<uint8_t *>(meta), nblk_max, teams};
    const bool e4m3 = fmt == SS_KV8_E4M3;
    auto *kernel = e4m3 ? write_of<SS_KV8_E4M3, kNoMeta>(blk) : write_of<SS_KV8_INT8, kNoMeta>(blk);
    if (meta && meta_kind == SS_META_CUBOID)
        kernel = e4m3 ? write_of<SS_KV8_E4M3, SS_META_CUBOID>(blk) : write_of<SS_KV8_INT8, SS_META_CUBOID>(blk);
    else if (meta)
        kernel = e4m3 ? write_of<SS_KV8_E4M3, SS_META_MEAN>(blk) : write_of<SS_KV8_INT8, SS_META_MEAN>(blk);
    ss::launch(kernel, dim3((unsigned)groups), dim3(kThreads), ss::as_stream(stream), a);
    return ss::check_launch("ss_write_kv8");
}

extern "C" ss_status ss_read_kv8(const void *kv_base, const int64_t *region_off, const int32_t *tables, int max_blocks,
                                 int32_t slot_limit, const void *open_blocks, const int32_t *len, const int32_t *row_begin,
                                 int B, int Hkv, int blk, int d, int rows, int fmt, void *k, void *v, int64_t row_stride,
                                 int64_t head_stride, void *stream)
{
    ss_status st = check_kv8("ss_read_kv8", B, Hkv, blk, d, fmt, slot_limit);
    if (st) return st;
    SS_CHECK_ARG(rows >= 0 && max_blocks >= 0, "ss_read_kv8: rows=%d max_blocks=%d", rows, max_blocks);
    SS_CHECK_ARG(row_stride >= 0 && head_stride >= 0 && row_stride % 16 == 0 && head_stride % 16 == 0,
                 "ss_read_kv8: strides %lld, %lld are no multiples of 16", (long long)row_stride, (long long)head_stride);
    if (B == 0 || rows == 0) return SS_OK;
    SS_CHECK_ARG(kv_base && region_off && open_blocks && len && row_begin && k && v, "ss_read_kv8: null pointer");
    SS_CHECK_ARG(aligned16(kv_base) && aligned16(open_blocks) && aligned16(k) && aligned16(v),
                 "ss_read_kv8: buffers must be 16-byte aligned");
    const int64_t teams = ((int64_t)B + rows / std::min(blk, 16)) * Hkv, groups = groups_of(teams, blk);
    SS_CHECK_SUPPORTED(groups <= 0x7FFFFFFF / kThreads, "ss_read_kv8: %lld block records pass the launch",
                       (long long)teams);
    const read_args a = {static_cast<const uint8_t *>(kv_base), region_off, tables, max_blocks, slot_limit,
                         static_cast<const uint8_t *>(open_blocks), len, row_begin, B, Hkv, rows, static_cast<uint8_t *>(k),
                         static_cast<uint8_t *>(v), row_stride, head_stride, teams};
    auto *kernel = fmt == SS_KV8_E4M3 ? read_of<SS_KV8_E4M3>(blk) : read_of<SS_KV8_INT8>(blk);
    ss::launch(kernel, dim3((unsigned)groups), dim3(kThreads), ss::as_stream(stream), a);
    return ss::check_launch("ss_read_kv8");
}
