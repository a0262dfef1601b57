// Decode attention over block records held in 8 bits (softmax(q K^T / sqrt(d)) V
// of Section 2.1 over the blocks of Section 2.2's selection, or over all of a
// sequence's blocks with its open block).
//
// As in attention.hip the query heads of a KV head are the 16 columns of the
// matrix products.  A wave takes 32 tokens (8 KiB of codes) a step:
//   S^T[2 x 16 tok x 16 heads] = K * Q^T     2 x 4 v_mfma_f32_16x16x32_f16
//   O^T[128 ch x 16 heads]    += V^T * P^T   8 x 2 v_mfma_f32_16x16x32_f16
// e4m3 and int8 codes are exact in f16, so they are widened in registers (int8
// by putting the byte into the low bits of 1024 + 128 + code) and the tiles'
// scales go where they cost one multiplication a token: K's into the logit, V's
// into the probability.  Queries become f16 by a power of two for each head,
// which leaves a channel off by at most 2^-39 of the largest; p * scale enters as
// two f16 parts, by a power of two for each head that follows the head's largest
// p * scale so far, which leaves a product off by at most 2^-23 of itself or 2^-35
// of that largest.  (A power of two for the largest scale alone, whatever its
// weight, let a tile of no weight take the others' bits: all of them beyond a
// scale of 2^35 times theirs.)  With bf16 operands and three parts a step took 211
// vector instructions, e4m3, and 340, int8; now 125 and 221.
// What p and its products are relative to stays as it is until one of them grows
// to kMost, so that most steps exchange nothing between lanes.
// The record's order of codes (kv8.hpp) makes a load instruction 1 KiB of
// consecutive bytes and leaves each lane with its own operand bytes, so
// nothing passes through LDS either:
//   lane (L = lane/16, col = lane%16) holds K of token `col` of a subtile,
//   16 channels a load; its accumulators are tokens 4L .. 4L+3 of both
//   subtiles, and those tokens' codes are its V operand, channels 8*col + t.
//
// HBM bounds it (256 bytes and a share of the trailer a token and head): 64
// sequences of 128 selected blocks of 16, 8 heads, take 45 us (6.2 TB/s), 16 of 8k
// to 64k tokens 194 us (6.5), one of 128k 47 to 56 us with its join, by where its
// records lie in memory (5.8 to 4.9; the kernel alone 45 to 51).  Each
// wave keeps two steps in flight; a CU has about 40 KB of loads in flight
// whatever the waves ask for (3 or 4 steps in flight gain nothing), so what
// counts is that all CUs have work.  Pages are resolved 64 entries at a time, an
// entry a lane, one set ahead, and read out as scalars.  A skipped entry reads
// a record of zeros, so the loads are unconditional; offsets are 64 bits.
//
// Work split: a workgroup's 4 waves take the steps of its range round-robin;
// their partials are merged through LDS and the parts of a unit that several
// workgroups took by a second kernel, both in a fixed order (plan() says who
// takes what).
#include <algorithm>
#include <cmath>

#include "kv8.hpp"

namespace {

constexpr int D = ss::kHeadDim;
constexpr int TOK = 32;  // tokens of a step
constexpr int WAVES = 4;
constexpr int CUS = 256;
constexpr int kShares = 512;  // workgroups of SHARE, two a CU
constexpr int kShareUnits = 16, kShareSteps = 224, kShareAll = 24576;  // from which they share (plan())
constexpr float kNone = -3e38f;  // the maximum of no tokens
constexpr float kMost = 32768.f;  // the largest p * scale (within f16's range) and sum of a step's p
constexpr int kTop = 10;          // to 2^kTop .. 2^(kTop + 1) the largest p * scale is taken anew
constexpr int kMaxSplits = 256;
constexpr int kMaxPartials = 4096;  // units * splits, where there is more than one split

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f4_t __attribute__((ext_vector_type(4), aligned(4)));  // the caller's floats
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

// Records are addressed as global memory explicitly: where the compiler lost
// that, it would wait for all loads in flight, the next step's among them.
typedef const uint8_t __attribute__((address_space(1))) *gptr_t;
template <class T>
__device__ __forceinline__ T load_stream(gptr_t p)
{
    return __builtin_nontemporal_load(reinterpret_cast<const T __attribute__((address_space(1))) *>(p));
}
template <class T>
__device__ __forceinline__ T load(gptr_t p)
{
    return *reinterpret_cast<const T __attribute__((address_space(1))) *>(p);
}

// what a skipped entry reads
__device__ __align__(128) unsigned char zero_record[ss::kv8_record(32)];

union frag_t {  // 8 x bf16 or f16
    bf16x8_t v;
    f16x8_t h;
    uint32_t w[4];
    u32x4_t u;
};

// four codes -> two registers of f16 (exact)
template <int FMT>
__device__ __forceinline__ void widen4(uint32_t c, uint32_t &a, uint32_t &b)
{
    if constexpr (FMT == SS_KV8_E4M3) {
        a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, 1.0f, false));
        b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, 1.0f, true));
    } else {
        // the bytes 128 + code become the low bits of 1024 + 128 + code
        const f16x2_t off = {(_Float16)-1152.f, (_Float16)-1152.f};
        c ^= 0x80808080u;
        a = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, c, 0x04010400)) + off);
        b = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, c, 0x04030402)) + off);
    }
}

// x minus the lower or upper f16 of h
__device__ __forceinline__ float minus_lo(uint32_t h, float x)
{
    asm("v_fma_mix_f32 %0, %1, -1.0, %0 op_sel_hi:[1,0,0]" : "+v"(x) : "v"(h));
    return x;
}
__device__ __forceinline__ float minus_hi(uint32_t h, float x)
{
    asm("v_fma_mix_f32 %0, %1, -1.0, %0 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "+v"(x) : "v"(h));
    return x;
}
// two floats as f16, rounded to nearest even
__device__ __forceinline__ uint32_t pack_f16(float x, float y)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{x, y}, f16x2_t));
}

// 1/x of a power of two between 2^-126 and 2^126
__device__ __forceinline__ float inverse(float x) { return __uint_as_float((254u << 23) - __float_as_uint(x)); }

// 127 and the exponent of a float of no sign
__device__ __forceinline__ int exponent(float x) { return (int)(__float_as_uint(x) >> 23); }

// maximum over the four 16-lane rows, in every lane
__device__ __forceinline__ float rows_max(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
}

// maximum over the wave, in every lane
__device__ __forceinline__ float wave_max(float x)
{
    auto f = [](float a, float b) { return fmaxf(a, b); };
    x = f(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xF, 0xF, false)));   // lane ^ 1
    x = f(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x4E, 0xF, 0xF, false)));   // lane ^ 2
    x = f(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x141, 0xF, 0xF, false)));  // mirrored in 8 lanes
    x = f(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x140, 0xF, 0xF, false)));  // mirrored in 16 lanes
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return f(__uint_as_float(h[0]), __uint_as_float(h[1]));
}

// a value that is the same in every lane, in scalar registers
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

struct attn_args {
    const uint16_t *q;
    const uint8_t *kv;
    const int64_t *region_off;
    const int32_t *sel, *tables;
    int max_blocks;
    const int32_t *capacity;
    int slot_limit;
    const int32_t *nblk;
    const uint8_t *open;
    const int32_t *len;
    int Hq, Hkv, G, k;
    float scale_log2;
    int B, per;  // per: steps of a split (SPLIT)
    float *out, *ws;
};

// entries that a unit of sequence b can have: all k, or without a selection its blocks
__device__ __forceinline__ int entries_of(const attn_args &a, int b)
{
    if (a.sel) return a.k;
    const int n = a.nblk[b];
    return n < 0 ? 0 : min(n, a.k);
}

// steps of a unit of sequence b, one at least
template <int BLK>
__device__ __forceinline__ uint32_t steps_of(const attn_args &a, int b)
{
    return max(1, (entries_of(a, b) * BLK + TOK - 1) / TOK);
}

// How the work is split.
//   SPLIT: grid (unit, split), each split a->per steps of its unit.
//   SHARE: the steps of all units stand in one line, unit after unit, and each
//   of the workgroups takes the same share of it, whatever the units' lengths
//   and however many there are (without a selection, where lengths differ).
// Where a unit's steps fall to several workgroups a second kernel joins them.
enum { SPLIT, SHARE };

// The line, found the same way by every wave of both kernels.
template <int BLK>
struct line_t {
    uint32_t total, share;
    uint32_t mine, upto;  // sequence `lane`: its steps for one head, and with those of the sequences before

    __device__ line_t(const attn_args &a, int lane)
    {
        mine = lane < a.B ? steps_of<BLK>(a, lane) : 0u;
        upto = ss::wave_scan_sum(mine);
        total = ss::lane_value(upto, 63);
        for (int b = 64; b < a.B; b += 64)
            total += ss::lane_value(ss::wave_scan_sum(b + lane < a.B ? steps_of<BLK>(a, b + lane) : 0u), 63);
        total *= (uint32_t)a.Hkv;
        share = ((total + kShares - 1) / kShares + WAVES - 1) / WAVES * WAVES;  // whole rounds of the waves
    }
    // the sequence of place x of the line, its steps for one head, and where it begins
    __device__ void find(const attn_args &a, int lane, uint32_t x, int &b, uint32_t &steps, uint32_t &begin) const
    {
        uint32_t n = mine, sum = upto, before = 0;
        for (int b0 = 0;;) {
            const unsigned long long past = __ballot((before + sum) * a.Hkv > x);
            if (past) {
                const int l = __builtin_ctzll(past);
                b = b0 + l;
                steps = ss::lane_value(n, l);
                begin = (before + ss::lane_value(sum, l) - steps) * a.Hkv;
                return;
            }
            before += ss::lane_value(sum, 63);
            b0 += 64;
            n = b0 + lane < a.B ? steps_of<BLK>(a, b0 + lane) : 0u;
            sum = ss::wave_scan_sum(n);
        }
    }
    // where sequence b begins
    __device__ uint32_t begin_of(const attn_args &a, int lane, int b) const
    {
        uint32_t before = 0;
        for (int b0 = 0; b0 < b; b0 += 64) {
            const int l = min(b - b0, 64) - 1;
            before += ss::lane_value(b0 ? ss::wave_scan_sum(b0 + lane < a.B ? steps_of<BLK>(a, b0 + lane) : 0u) : upto, l);
        }
        return before * a.Hkv;
    }
};

// Floats of a part of one head: maximum, sum, output.  SPLIT has room for a part
// of each split, SHARE for two of each share (of its first unit, which may
// have begun before, and of its last).
constexpr int64_t kPartHead = D + 2;

template <int BLK, int FMT, int MODE>
__global__ __launch_bounds__(WAVES * 64, MODE == SPLIT ? 3 : 2) void attn_kv8_kernel(const attn_args a)
{
    constexpr int REC = ss::kv8_record(BLK), OPEN = 2 * BLK * D * 2;
    constexpr int EPS = TOK / BLK;        // entries of a step
    constexpr int SET = 64 / EPS;         // steps of a set of 64 entries
    // the waves' partial results, and that of the open record
    __shared__ float sm_m[WAVES + 1][16], sm_l[WAVES + 1][16], sm_g[WAVES + 1][16];
    __shared__ __align__(16) float sm_o[WAVES + 1][16][D + 4];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int L = lane >> 4, col = lane & 15;
    int b, u;                 // sequence and unit
    int nsteps, first, last;  // the unit's steps, and the range taken here
    uint32_t at_step = 0, end_step = 0, begin_step = 0;  // on the line
    if (MODE == SHARE) {
        const line_t<BLK> line(a, lane);
        begin_step = blockIdx.x * line.share;
        if (begin_step >= line.total) return;
        uint32_t steps, begin;
        line.find(a, lane, begin_step, b, steps, begin);
        // the same in every lane, which the compiler does not see
        b = __builtin_amdgcn_readfirstlane(b);
        nsteps = __builtin_amdgcn_readfirstlane(steps);
        begin = __builtin_amdgcn_readfirstlane(begin);
        at_step = begin_step = __builtin_amdgcn_readfirstlane(begin_step);
        end_step = __builtin_amdgcn_readfirstlane(min(begin_step + line.share, line.total));
        const int g = (int)((at_step - begin) / (uint32_t)nsteps);
        u = b * a.Hkv + g;
        first = (int)(at_step - begin) - g * nsteps;
        last = min(nsteps, first + (int)(end_step - at_step));
    } else {
        u = blockIdx.x;
        b = u / a.Hkv;
        nsteps = (int)steps_of<BLK>(a, b);
        first = blockIdx.y * a.per;
        last = min(first + a.per, nsteps);
        if (first >= nsteps) return;
    }

    for (;;) {
        const int g = u - b * a.Hkv;
        const int n_entries = entries_of(a, b);
        const int s_begin = first, s_end = last;
        const int open_rows = a.open ? __builtin_amdgcn_readfirstlane(max(a.len[b], 0) & (BLK - 1)) : 0;
        const bool tail = first == 0 && open_rows > 0;

        // B operand of S^T: head `col`, channels 64*(m/2) + 16L + 8*(m%2) .. +7
        frag_t qf[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const int h = col < a.G ? col : 0;
            const uint16_t *qh = a.q + ((int64_t)b * a.Hq + g * a.G + h) * D;
            const u32x4_t w = *reinterpret_cast<const u32x4_t *>(qh + 64 * (m >> 1) + 16 * L + 8 * (m & 1));
            qf[m].u = col < a.G ? w : u32x4_t{0, 0, 0, 0};
        }

        const gptr_t base = (gptr_t)(a.kv + uniform(a.region_off[u]));
        int limit = a.slot_limit;
        if (a.capacity) limit = min(limit, a.capacity[u]);
        const int blocks = a.nblk ? a.nblk[b] : 0x7FFFFFFF;
        // the page of entry i of the wave's steps from step `first` on, a lane each.
        // What bounds an entry by the sequence's length is applied last, so that no
        // load waits for the length.
        auto resolve = [&](int first) {
            const int st = first + (lane / EPS) * WAVES, e = st * EPS + lane % EPS;
            int block = -1, page = -1;
            if (e < a.k) block = a.sel ? a.sel[(int64_t)u * a.k + e] : e;
            if (!a.tables) page = block;
            else if (block >= 0 && block < a.max_blocks) page = a.tables[(int64_t)b * a.max_blocks + block];
            return st < s_end && e < n_entries && block < blocks && page < limit ? page : -1;
        };

        // Softmax state of head `col`: mref, a whole number that p is relative to;
        // lrun, the lane's sum of p; gain, a power of two that the V scales are
        // multiplied by, so that p * scale is in f16's range and the largest so
        // far at least 2^kTop.
        float mref = kNone, lrun = 0.f, gain = 0x1p126f;
        f32x4_t o[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) o[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        // a partial result to LDS; the lane holds channels 32L + 8i + t of head `col`.
        // mref may lie far below the largest logit, so the sum is taken to [1, 2):
        // the outputs are then of V's size.
        auto put = [&](int place) {
            float l = lrun + __shfl_xor(lrun, 16);
            l += __shfl_xor(l, 32);
            const int e = place < WAVES ? max(exponent(l) - 127, 0) : 0;
            if (L == 0) {
                sm_m[place][col] = mref + (float)e;
                sm_l[place][col] = __builtin_ldexpf(l, -e);
                sm_g[place][col] = __builtin_ldexpf(1.f, 127 - exponent(gain) - e);
            }
            if (col < a.G) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float *row = &sm_o[place][col][32 * L + 8 * i];
                    *reinterpret_cast<f32x4_t *>(row) = f32x4_t{o[0][i], o[1][i], o[2][i], o[3][i]};
                    *reinterpret_cast<f32x4_t *>(row + 4) = f32x4_t{o[4][i], o[5][i], o[6][i], o[7][i]};
                }
            }
        };

        gptr_t zeros = (gptr_t)zero_record;
        asm("" : "+s"(zeros));  // its address is looked up once
        struct step_t {
            u32x4_t k[4], v[4];  // subtile 0, 1; channels 0..63, 64..127 (K), channel quads (V)
            f32x2_t sc[2];       // scales of the lane's accumulator tokens
            bool ok[2];
        };
        auto load_step = [&](const int (&page)[EPS], step_t &x) {
            gptr_t rec[EPS];
#pragma unroll
            for (int e = 0; e < EPS; ++e) {
                // both addresses first: a branch would hold the loads back
                gptr_t r = base + (int64_t)page[e] * REC;
                asm("" : "+s"(r));
                rec[e] = page[e] >= 0 ? r : zeros;
            }
            auto get = [](gptr_t p) { return load_stream<u32x4_t>(p); };
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if constexpr (BLK == 8) {
                    const bool kw = col >> 3, vw = L >> 1;  // which of the subtile's two records
                    const gptr_t kr = (kw ? rec[2 * s + 1] : rec[2 * s]) + L * 128 + (col & 7) * 16;
                    const gptr_t r = vw ? rec[2 * s + 1] : rec[2 * s];
                    const gptr_t vr = r + BLK * D + (L & 1) * 256 + col * 16;
                    x.k[2 * s] = get(kr);
                    x.k[2 * s + 1] = get(kr + 512);
                    x.v[2 * s] = get(vr);
                    x.v[2 * s + 1] = get(vr + 512);
                    x.sc[s] = load<f32x2_t>(r + 2 * BLK * D);
                    x.ok[s] = (vw ? page[2 * s + 1] : page[2 * s]) >= 0;
                } else {
                    constexpr int PER = BLK / 16;  // subtiles of a record
                    const gptr_t r = rec[s / PER] + lane * 16;
                    x.k[2 * s] = get(r + (s % PER) * 2048);
                    x.k[2 * s + 1] = get(r + (s % PER) * 2048 + 1024);
                    x.v[2 * s] = get(r + BLK * D + (s % PER) * 2048);
                    x.v[2 * s + 1] = get(r + BLK * D + (s % PER) * 2048 + 1024);
                    x.sc[s] = load<f32x2_t>(rec[s / PER] + 2 * BLK * D);
                    x.ok[s] = page[s / PER] >= 0;
                }
            }
        };
        float q_scale = 0.f;  // turns the products of f16 queries into logits (exp2 domain)
        auto compute_step = [&](const step_t &x) {
            f32x4_t acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    frag_t f;
                    widen4<FMT>(x.k[2 * s + (m >> 1)][2 * (m & 1)], f.w[0], f.w[1]);
                    widen4<FMT>(x.k[2 * s + (m >> 1)][2 * (m & 1) + 1], f.w[2], f.w[3]);
                    acc[s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f.h, qf[m].h, acc[s], 0, 0, 0);
                }
            const float sk[2] = {x.ok[0] ? x.sc[0].x * q_scale : 0.f, x.ok[1] ? x.sc[1].x * q_scale : 0.f};
            float p[8], v[8], sum, top;  // probabilities, times V scales and gain; their sum and the largest of both
            auto weigh = [&] {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const float bias = x.ok[s] ? -mref : -INFINITY, sv = x.sc[s].y * gain;
#pragma unroll
                    for (int i = 4 * s; i < 4 * s + 4; ++i) {
                        p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[s][i & 3], sk[s], bias));
                        v[i] = p[i] * sv;
                    }
                }
                sum = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
                top = sum;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, v[i]);
            };
            weigh();
            if (__builtin_expect(__any(top > kMost), 0)) {
                float z[2], y = 0.f;  // the subtiles' largest logits; the largest product
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    z[s] = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[s] = fmaxf(z[s], x.ok[s] ? acc[s][i] * sk[s] : -INFINITY);
                }
                // whole numbers, so that what is there is rescaled exactly, and not at all
                // where its largest product stays the largest
                const float mnew = fmaxf(mref, __builtin_ceilf(rows_max(fmaxf(z[0], z[1]))));
                const int rise = (int)fminf(mnew - mref, 1024.f);
#pragma unroll
                for (int s = 0; s < 2; ++s) y = fmaxf(y, __builtin_amdgcn_exp2f(z[s] - mnew) * x.sc[s].y);
                const int gnew = min(min(exponent(gain) + rise, 253), 254 + kTop - exponent(rows_max(y)));
                const float f = __builtin_ldexpf(1.f, gnew - exponent(gain) - rise);
#pragma unroll
                for (int t = 0; t < 8; ++t) o[t] *= f;
                lrun = __builtin_ldexpf(lrun, -rise);
                mref = mnew;
                gain = __uint_as_float((uint32_t)gnew << 23);
                weigh();
            }
            lrun += sum;
            frag_t hi, lo;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                hi.w[i >> 1] = pack_f16(v[i], v[i + 1]);
                lo.w[i >> 1] = pack_f16(minus_lo(hi.w[i >> 1], v[i]), minus_hi(hi.w[i >> 1], v[i + 1]));
            }
            // four accumulators in turn, so that none waits for its last product
#pragma unroll
            for (int t = 0; t < 8; t += 4) {
                frag_t w[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    widen4<FMT>(x.v[t >> 2][h], w[h].w[0], w[h].w[1]);
                    widen4<FMT>(x.v[2 + (t >> 2)][h], w[h].w[2], w[h].w[3]);
                }
#pragma unroll
                for (int h = 0; h < 4; ++h) o[t + h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w[h].h, hi.h, o[t + h], 0, 0, 0);
#pragma unroll
                for (int h = 0; h < 4; ++h) o[t + h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w[h].h, lo.h, o[t + h], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        };

        int st = s_begin + wave;
        int pages = resolve(st), ahead = -1;
        if (s_end - s_begin > SET * WAVES) ahead = resolve(st + SET * WAVES);
        int at = 0, later = st + 2 * SET * WAVES;  // the next step's place in the set; the set after `ahead`
        auto load_next = [&](step_t &x) {
            int page[EPS];
#pragma unroll
            for (int e = 0; e < EPS; ++e) page[e] = __builtin_amdgcn_readlane(pages, at * EPS + e);
            load_step(page, x);
            if (__builtin_expect(++at == SET, 0)) {
                at = 0;
                pages = ahead;
                ahead = resolve(later);
                later += SET * WAVES;
            }
        };

        // The open record, a partial result of its own: bf16 rows of K,
        // channel-major V, and p as three bf16 parts; rows past the last are not
        // read.  All of it is on its way before the first step's codes (read where
        // it is used, it added 8 us to 46 of a sequence of 128k tokens).
        constexpr int OS = BLK == 32 ? 2 : 1;  // its subtiles
        u32x4_t open_k[4 * OS];
        u32x2_t open_v[8 * OS];
        const bool opens = tail && wave == WAVES - 1;
        if (opens) {
            const uint8_t *ok = a.open + (int64_t)u * OPEN, *ov = ok + BLK * D * 2;
#pragma unroll
            for (int i = 0; i < 4 * OS; ++i) {
                const int tok = 16 * (i >> 2) + col, ch = 64 * (i >> 1 & 1) + 16 * L + 8 * (i & 1);
                open_k[i] = u32x4_t{0, 0, 0, 0};
                if (tok < open_rows) open_k[i] = *reinterpret_cast<const u32x4_t *>(ok + (tok * D + ch) * 2);
            }
#pragma unroll
            for (int i = 0; i < 8 * OS; ++i) {
                const int tok = 16 * (i >> 3) + 4 * L;
                open_v[i] = u32x2_t{0, 0};
                if (tok < open_rows) open_v[i] = *reinterpret_cast<const u32x2_t *>(ov + ((8 * col + (i & 7)) * BLK + tok) * 2);
            }
        }

        step_t bufA, bufB;
        load_next(bufA);

        if (opens) {
            float z[8], cm = kNone;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    frag_t f;
                    f.u = s < OS ? open_k[4 * (s % OS) + m] : u32x4_t{0, 0, 0, 0};
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.v, qf[m].v, acc, 0, 0, 0);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    z[4 * s + i] = 16 * s + 4 * L + i < open_rows ? acc[i] * a.scale_log2 : -INFINITY;
                    cm = fmaxf(cm, z[4 * s + i]);
                }
            }
            mref = rows_max(cm);
            gain = 1.f;
            frag_t part[3];
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                float x0 = __builtin_amdgcn_exp2f(z[i] - mref), x1 = __builtin_amdgcn_exp2f(z[i + 1] - mref);
                lrun += x0;
                lrun += x1;
#pragma unroll
                for (int j = 0; j < 3; ++j) {  // each takes the upper half of what is left
                    const uint32_t w = __builtin_amdgcn_perm(__float_as_uint(x1), __float_as_uint(x0), 0x07060302);
                    part[j].w[i >> 1] = w;
                    x0 -= __uint_as_float(w << 16);
                    x1 -= __uint_as_float(w & 0xFFFF0000u);
                }
            }
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                frag_t f;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const int left = open_rows - 16 * s - 4 * L;  // the lane's live tokens
                    const u32x2_t w = s < OS ? open_v[8 * (s % OS) + t] : u32x2_t{0, 0};
                    f.w[2 * s] = left > 1 ? w.x : w.x & 0xFFFFu;
                    f.w[2 * s + 1] = left > 3 ? w.y : left > 2 ? w.y & 0xFFFFu : 0u;
                }
#pragma unroll
                for (int j = 0; j < 3; ++j) o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.v, part[j].v, o[t], 0, 0, 0);
            }
            put(WAVES);
            mref = kNone;
            lrun = 0.f;
            gain = 0x1p126f;
#pragma unroll
            for (int t = 0; t < 8; ++t) o[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }

        // the queries as f16, times a power of two that takes the head's largest
        // to [2^14, 2^15): bf16's 8 bits fit down to 2^-31 of it, one down to 2^-38
        {
            uint32_t mag = 0;
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    mag = max(mag, max(qf[m].w[i] << 16 & 0x7FFF0000u, qf[m].w[i] & 0x7FFF0000u));
            const int e = exponent(rows_max(__uint_as_float(min(mag, 0x7F800000u))));
            const int to = min(254 + 14 - e, 253);
            const float up = __uint_as_float((uint32_t)to << 23);
            // with an infinity or a NaN among them every logit is NaN (and no skipped entry's)
            const bool fine = e < 255;
            q_scale = fine ? a.scale_log2 * inverse(up) : __uint_as_float(0x7FC00000u);
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t w = qf[m].w[i];
                    qf[m].w[i] = fine ? pack_f16(__uint_as_float(w << 16) * up, __uint_as_float(w & 0xFFFF0000u) * up) : 0u;
                }
        }

        for (; st < s_end; st += 2 * WAVES) {
            load_next(bufB);
            compute_step(bufA);
            if (st + WAVES >= s_end) break;
            load_next(bufA);
            compute_step(bufB);
        }
        put(wave);
        // the open tokens' too: the infinities that they may have got have no softmax,
        // whatever their signs
        if (opens && L == 0 && q_scale != q_scale) sm_l[WAVES][col] = q_scale;
        __syncthreads();
        const int partials = tail ? WAVES + 1 : WAVES;
        for (int idx = threadIdx.x; idx < a.G * (D / 4); idx += WAVES * 64) {
            const int h = idx / (D / 4), ch = idx % (D / 4) * 4;
            float M = kNone;
            for (int w = 0; w < partials; ++w) M = fmaxf(M, sm_m[w][h]);
            float lsum = 0.f;
            f32x4_t osum = {0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < partials; ++w) {
                const float sc = __builtin_amdgcn_exp2f(sm_m[w][h] - M);
                lsum += sc * sm_l[w][h];
                osum += sc * sm_g[w][h] * *reinterpret_cast<const f32x4_t *>(&sm_o[w][h][ch]);
            }
            if (first == 0 && last == nsteps) {
                if (lsum != 0.f) osum /= lsum;
                *reinterpret_cast<f4_t *>(a.out + ((int64_t)b * a.Hq + g * a.G + h) * D + ch) = osum;
            } else {
                const int64_t place = MODE == SHARE ? (int64_t)blockIdx.x * 2 + (at_step == begin_step ? 0 : 1)
                                                    : (int64_t)u * gridDim.y + blockIdx.y;
                float *pp = a.ws + (place * a.G + h) * kPartHead;
                if (ch == 0) {
                    pp[0] = M;
                    pp[1] = lsum;
                }
                *reinterpret_cast<f4_t *>(pp + 2 + ch) = osum;
            }
        }
        if (MODE == SPLIT) return;
        at_step += last - first;
        if (at_step >= end_step) return;
        ++u;
        first = 0;
        if (u - b * a.Hkv == a.Hkv) {
            ++b;
            nsteps = __builtin_amdgcn_readfirstlane((int)steps_of<BLK>(a, b));
        }
        last = min(nsteps, (int)(end_step - at_step));
        __syncthreads();  // the partials in LDS have been read
    }
}

// Joins the parts of the units whose steps fell to several workgroups, in their
// order: one workgroup per (unit, head), two channels a lane, 8 parts a wave
// at a time, all read at once beside their maxima and sums.
template <int BLK, int W, int MODE>
__global__ __launch_bounds__(W * 64) void join_kv8_kernel(const attn_args a, int splits)
{
    typedef float f2_t __attribute__((ext_vector_type(2), aligned(4)));
    __shared__ float s_m[W], s_l[W];
    __shared__ f32x2_t s_o[W][64];
    const int u = blockIdx.x, h = blockIdx.y, lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int b = u / a.Hkv, g = u - b * a.Hkv;
    const uint32_t steps = steps_of<BLK>(a, b);
    uint32_t parts;
    int64_t place0, place1;  // of the first part and the second; the others follow at the same distance
    if (MODE == SHARE) {
        const line_t<BLK> line(a, lane);
        const uint32_t begin = line.begin_of(a, lane, b) + (uint32_t)g * steps, w0 = begin / line.share;
        parts = (begin + steps - 1) / line.share - w0 + 1;
        place0 = 2 * (int64_t)w0 + (begin != w0 * line.share ? 1 : 0);
        place1 = 2 * (int64_t)w0 + 2;
    } else {
        parts = (steps + a.per - 1) / a.per;
        place0 = (int64_t)u * splits;
        place1 = place0 + 1;
    }
    if (parts == 1) return;  // written by its one workgroup
    auto part = [&](uint32_t i) {
        return a.ws + ((i ? place1 + (int64_t)(i - 1) * (MODE == SHARE ? 2 : 1) : place0) * a.G + h) * kPartHead;
    };
    float M = -INFINITY, lsum = 0.f;
    f32x2_t osum = {0.f, 0.f};
    for (uint32_t p0 = wave * 8; p0 < parts; p0 += W * 8) {
        f2_t x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const f2_t *>(part(min(p0 + i, parts - 1)) + 2 + 2 * lane);
        f2_t ml = {-INFINITY, 0.f};
        if (lane < 8 && p0 + lane < parts) ml = *reinterpret_cast<const f2_t *>(part(p0 + lane));
        const float mnew = fmaxf(M, wave_max(ml.x)), m0 = mnew == -INFINITY ? 0.f : mnew;
        const float alpha = __builtin_amdgcn_exp2f(M - m0), w = __builtin_amdgcn_exp2f(ml.x - m0);
        lsum *= alpha;
        osum *= alpha;
        M = mnew;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // a part of weight 0 counts, for the NaN that it may hold
            const float sc = __uint_as_float(ss::lane_value(__float_as_uint(w), i));
            if (p0 + i < parts) {
                lsum += sc * __uint_as_float(ss::lane_value(__float_as_uint(ml.y), i));
                osum.x += sc * x[i].x;
                osum.y += sc * x[i].y;
            }
        }
    }
    if (W > 1) {
        s_o[wave][lane] = osum;
        if (lane == 0) {
            s_m[wave] = M;
            s_l[wave] = lsum;
        }
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int j = 1; j < W; ++j) M = fmaxf(M, s_m[j]);
        const float m0 = M == -INFINITY ? 0.f : M;
        lsum = 0.f;
        osum = f32x2_t{0.f, 0.f};
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const float sc = __builtin_amdgcn_exp2f(s_m[j] - m0);
            lsum += sc * s_l[j];
            osum.x += sc * s_o[j][lane].x;
            osum.y += sc * s_o[j][lane].y;
        }
    }
    f2_t y = {0.f, 0.f};
    if (lsum != 0.f) y = f2_t{osum.x / lsum, osum.y / lsum};
    *reinterpret_cast<f2_t *>(a.out + ((int64_t)b * a.Hq + g * a.G + h) * D + 2 * lane) = y;
}

struct split_plan {
    int mode, splits, per;
};

// SHARE where a call attends to all blocks of sequences whose lengths only the
// GPU knows, and there is enough work to make up for its longer start (about 3
// us: the line, a second unit begun within a share, the join).  us, SPLIT and
// SHARE, lengths from an eighth of the longest on: 16 units of up to 2048 steps
// 37.7, 32.3; 96 of 256 30.5, 25.1; 128 of 256 33.4, 33.1; 512 of 300 124, 116.
// Less work: 64 of 320 25.3, 28.8; 16 of 1024 23.9, 27.5; short units, of which
// a share has several: 162 of 126 24.9, 28.7; 614 of 170 95, 109.  Over 275
// shapes of 8 to 624 units, 91 to 4096 steps, these three lines lose 0.9%
// against the better of both on average, 14% at most; SPLIT alone 4% and 40%.
//
// SPLIT takes the splits that cost least by a model of the time (us; fitted to
// 1875 shapes of 1 to 1024 units, 1 to 4096 steps, G 1 to 16, each block size
// and format: its choices lose 0.8% against the best on average, three
// workgroups a CU lose 5%, up to 50%):
//   - the chip's bandwidth: kStepHbm a step;
//   - the fullest CU: a workgroup's waves take a step each per round, of
//     kRound1 alone on the CU, kRound2 beside another, kRound3 for each of more;
//     kGroup a workgroup besides;
//   - the join, a second launch.
// The ranges follow from k, not from the lengths: 8k tokens of one request, 8
// heads, blocks of 16, take 10.1 us with k = 513, 12.6 with 2048 and 24.3 with
// 8192, where two of 32 splits have work (of eight requests 25.7 and 26.2).
split_plan plan(int64_t units, int k, int blk, int G, bool selected, size_t room)
{
    const int steps = (int)(((int64_t)k * blk + TOK - 1) / TOK);
    const int64_t all = units * steps;
    const size_t part = G * kPartHead * sizeof(float);
    if (!selected && units >= kShareUnits && steps >= kShareSteps && all >= kShareAll && all <= 0x7FFFFFFF &&
        room >= 2 * kShares * part)
        return {SHARE, kShares, 0};
    constexpr float kStepHbm = 0.00096f, kRound1 = 0.73f, kRound2 = 1.6f, kRound3 = 0.84f, kGroup = 0.2f, kBoth = 0.088f;
    constexpr float kJoin = 2.61f, kJoinSplit = 0.012f, kJoinGroup = 0.00045f, kJoinHead = 0.00012f;
    const int64_t most = std::min<int64_t>(std::min<int64_t>(kMaxSplits, room / part / units), kMaxPartials / units);
    int best = 1;
    float least = 0.f;
    for (int n = 1; n == 1 || (n <= most && n <= steps); ++n) {
        const int per = (steps + n - 1) / n, splits = (steps + per - 1) / per;
        if (n > 1 && splits < n) continue;  // the same as with fewer
        const float groups = (float)units * splits, fullest = std::ceil(groups / CUS);
        const float rounds = (float)((per + WAVES - 1) / WAVES);
        const float hbm = all * kStepHbm;
        const float cu = rounds * (fullest == 1.f ? kRound1 : fullest == 2.f ? kRound2 : kRound3 * fullest) + kGroup * fullest;
        float cost = std::max(hbm, cu) + kBoth * std::min(hbm, cu);
        if (splits > 1) cost += kJoin + kJoinSplit * splits + (kJoinGroup + kJoinHead * G) * groups;
        if (n == 1 || cost < least) {
            best = n;
            least = cost;
        }
    }
    const int per = (steps + best - 1) / best;
    return {SPLIT, (steps + per - 1) / per, per};
}

bool has_plan(int B, int Hq, int Hkv, int d, int blk, int k)
{
    return B > 0 && Hkv > 0 && Hq > 0 && Hq % Hkv == 0 && d == D && ss::supported_blk(blk) && k > 0;
}

// bytes of a plan's parts
size_t plan_bytes(const split_plan &p, int64_t units, int G)
{
    const size_t part = G * kPartHead * sizeof(float);
    return p.mode == SHARE ? 2 * kShares * part : p.splits > 1 ? units * p.splits * part : 0;
}

template <int BLK>
auto join_of(int mode, int waves)
{
    if (mode == SHARE) return join_kv8_kernel<BLK, 8, SHARE>;
    if (waves == 1) return join_kv8_kernel<BLK, 1, SPLIT>;
    return waves == 4 ? join_kv8_kernel<BLK, 4, SPLIT> : join_kv8_kernel<BLK, 8, SPLIT>;
}

template <int FMT, int MODE>
auto attn_of(int blk)
{
    return blk == 8 ? attn_kv8_kernel<8, FMT, MODE> : blk == 16 ? attn_kv8_kernel<16, FMT, MODE> : attn_kv8_kernel<32, FMT, MODE>;
}

}  // namespace

extern "C" size_t ss_sparse_attention_kv8_workspace(int B, int Hq, int Hkv, int d, int blk, int k)
{
    if (!has_plan(B, Hq, Hkv, d, blk, k)) return 0;
    // what a call takes depends on whether it selects: room for either
    const int64_t units = (int64_t)B * Hkv;
    const int G = Hq / Hkv;
    const size_t any = ~(size_t)0 >> 1;
    return std::max(plan_bytes(plan(units, k, blk, G, false, any), units, G),
                    plan_bytes(plan(units, k, blk, G, true, any), units, G));
}

extern "C" ss_status ss_sparse_attention_kv8(const void *q, const void *kv_base, const int64_t *region_off,
                                             const int32_t *sel, const int32_t *tables, int max_blocks,
                                             const int32_t *capacity, int32_t slot_limit, const int32_t *nblk,
                                             const void *open_blocks, const int32_t *len, int fmt, int B, int Hq, int Hkv,
                                             int d, int blk, int k, float scale, float *out, void *workspace,
                                             size_t ws_bytes, void *stream)
{
    SS_CHECK_ARG(B >= 0 && Hq > 0 && Hkv > 0 && k > 0 && max_blocks >= 0 && slot_limit >= 0,
                 "ss_sparse_attention_kv8: bad shape B=%d Hq=%d Hkv=%d k=%d max_blocks=%d slot_limit=%d", B, Hq, Hkv, k,
                 max_blocks, slot_limit);
    SS_CHECK_ARG(Hq % Hkv == 0, "ss_sparse_attention_kv8: Hq=%d not a multiple of Hkv=%d", Hq, Hkv);
    SS_CHECK_ARG(fmt == SS_KV8_E4M3 || fmt == SS_KV8_INT8, "ss_sparse_attention_kv8: format %d", fmt);
    SS_CHECK_SUPPORTED(Hq / Hkv <= ss::kMaxGroup, "ss_sparse_attention_kv8: group size %d > %d", Hq / Hkv, ss::kMaxGroup);
    SS_CHECK_SUPPORTED(d == D, "ss_sparse_attention_kv8: d=%d (only 128)", d);
    SS_CHECK_SUPPORTED(ss::supported_blk(blk), "ss_sparse_attention_kv8: blk=%d (8, 16 or 32)", blk);
    SS_CHECK_SUPPORTED(k <= ss::kMaxBlocks, "ss_sparse_attention_kv8: k=%d > %d", k, ss::kMaxBlocks);
    SS_CHECK_ARG(std::isfinite(scale), "ss_sparse_attention_kv8: scale not finite");
    SS_CHECK_ARG(sel || nblk || B == 0, "ss_sparse_attention_kv8: without a selection the block counts are needed");
    SS_CHECK_ARG((open_blocks == nullptr) == (len == nullptr), "ss_sparse_attention_kv8: open blocks and lengths come together");
    if (B == 0) return SS_OK;
    SS_CHECK_ARG(q && kv_base && region_off && out, "ss_sparse_attention_kv8: null pointer");
    SS_CHECK_ARG((((uintptr_t)q | (uintptr_t)kv_base | (uintptr_t)open_blocks) & 15) == 0,
                 "ss_sparse_attention_kv8: buffers must be 16-byte aligned");
    const int64_t units = (int64_t)B * Hkv;
    SS_CHECK_SUPPORTED(units <= 0x7FFFFFFF / (WAVES * 64), "ss_sparse_attention_kv8: %lld units pass the launch",
                       (long long)units);
    const int G = Hq / Hkv;
    const split_plan sp = plan(units, k, blk, G, sel != nullptr, workspace ? ws_bytes : 0);
    const attn_args a = {static_cast<const uint16_t *>(q), static_cast<const uint8_t *>(kv_base), region_off, sel, tables,
                         max_blocks, capacity, slot_limit, nblk, static_cast<const uint8_t *>(open_blocks), len, Hq, Hkv, G,
                         k, scale * 1.4426950408889634f, B, sp.per, out, static_cast<float *>(workspace)};
    hipStream_t s = ss::as_stream(stream);
    const bool e4m3 = fmt == SS_KV8_E4M3;
    auto *kernel = e4m3 ? attn_of<SS_KV8_E4M3, SPLIT>(blk) : attn_of<SS_KV8_INT8, SPLIT>(blk);
    if (sp.mode == SHARE) kernel = e4m3 ? attn_of<SS_KV8_E4M3, SHARE>(blk) : attn_of<SS_KV8_INT8, SHARE>(blk);
    const dim3 grid = sp.mode == SHARE ? dim3(kShares) : dim3((unsigned)units, sp.splits);
    ss::launch(kernel, grid, dim3(WAVES * 64), s, a);
    ss_status st = ss::check_launch("ss_sparse_attention_kv8");
    if (st != SS_OK || sp.splits == 1) return st;
    const int waves = sp.mode == SHARE || sp.splits > 32 ? 8 : sp.splits > 8 ? 4 : 1;  // 8 parts each
    auto *join = blk == 8 ? join_of<8>(sp.mode, waves) : blk == 16 ? join_of<16>(sp.mode, waves) : join_of<32>(sp.mode, waves);
    join<<<dim3((unsigned)units, G), dim3(waves * 64), 0, s>>>(a, sp.splits);
    return ss::check_launch("ss_sparse_attention_kv8(join)");
}
