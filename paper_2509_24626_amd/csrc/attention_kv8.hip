// Decode attention over block records held in 8 bits (softmax(q K^T / sqrt(d)) V
// of Section 2.1 over the blocks of Section 2.2's selection, or over all of a
// sequence's blocks with its open block).
//
// As in attention.hip the query heads of a KV head are the 16 columns of the
// matrix products.  A wave takes 32 tokens (8 KiB of codes) a step:
//   S^T[2 x 16 tok x 16 heads] = K * Q^T     2 x 4 v_mfma_f32_16x16x32_bf16
//   O^T[128 ch x 16 heads]    += V^T * P^T   8 x 3 v_mfma_f32_16x16x32_bf16
// e4m3 and int8 codes are exact in bf16, so they are widened in registers and
// the tiles' scales go where they cost one multiplication a token: K's into
// the logit, V's into the probability.  P then enters the product as three
// bf16 parts (24 bits; two lose the last 8 and showed as 1e-5 in the output).
// The record's order of codes (kv8.hpp) makes a load instruction 1 KiB of
// consecutive bytes and leaves each lane with its own operand bytes, so
// nothing passes through LDS or between lanes:
//   lane (L = lane/16, col = lane%16) holds K of token `col` of a subtile,
//   16 channels a load; its accumulators are tokens 4L .. 4L+3 of both
//   subtiles, and those tokens' codes are its V operand, channels 8*col + t.
//
// HBM bounds it (256 bytes and a share of the trailer a token and head).  Each
// wave keeps two steps in flight.  Pages are resolved 64 entries at a time, an
// entry a lane, one set ahead, and read out as scalars.  A skipped entry reads
// a record of zeros, so the loads are unconditional; offsets are 64 bits.
//
// Work split: grid (unit, split), 4 waves taking steps round-robin over the
// split's range; wave partials are merged through LDS and splits by a second
// kernel, both in a fixed order.
#include <algorithm>
#include <cmath>

#include "kv8.hpp"

namespace {

constexpr int D = ss::kHeadDim;
constexpr int TOK = 32;  // tokens of a step
constexpr int WAVES = 4;
constexpr int CUS = 256;
constexpr int kMaxSplits = 256;
constexpr int kMaxPartials = 4096;  // units * splits, where there is more than one split

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

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

union frag_t {  // 8 x bf16
    bf16x8_t v;
    uint32_t w[4];
    u32x4_t u;
};

// four codes -> two registers of bf16 (exact)
template <int FMT>
__device__ __forceinline__ void widen4(uint32_t c, uint32_t &a, uint32_t &b)
{
    if constexpr (FMT == SS_KV8_E4M3) {
        a = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, 1.0f, false));
        b = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c, 1.0f, true));
    } else {
        const float x = (float)(int8_t)c, y = (float)(int8_t)(c >> 8), z = (float)(int8_t)(c >> 16), w = (float)(int8_t)(c >> 24);
        a = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302);
        b = __builtin_amdgcn_perm(__float_as_uint(w), __float_as_uint(z), 0x07060302);
    }
}

// maximum over the four 16-lane rows, in every lane
__device__ __forceinline__ float rows_max(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
}

// over all lanes, in every lane and in a fixed order
template <class F>
__device__ __forceinline__ float wave_fold(float x, const F &f)
{
    x = f(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xF, 0xF, false)));   // lane ^ 1
    x = f(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x4E, 0xF, 0xF, false)));   // lane ^ 2
    x = f(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x141, 0xF, 0xF, false)));  // mirrored in 8 lanes
    x = f(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x140, 0xF, 0xF, false)));  // mirrored in 16 lanes
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return f(__uint_as_float(h[0]), __uint_as_float(h[1]));
}
__device__ __forceinline__ float wave_max(float x) { return wave_fold(x, [](float a, float b) { return fmaxf(a, b); }); }
__device__ __forceinline__ float wave_sum(float x) { return wave_fold(x, [](float a, float b) { return a + b; }); }

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
    int steps_per_split;
    float *out, *ws;
};

// entries that unit u's sequence b can have: all k, or without a selection its blocks
__device__ __forceinline__ int entries_of(const attn_args &a, int b)
{
    if (a.sel) return a.k;
    const int n = a.nblk[b];
    return n < 0 ? 0 : min(n, a.k);
}

template <int BLK, int FMT>
__global__ __launch_bounds__(WAVES * 64, 3) void attn_kv8_kernel(const attn_args a)
{
    constexpr int REC = ss::kv8_record(BLK), OPEN = 2 * BLK * D * 2;
    constexpr int EPS = TOK / BLK;        // entries of a step
    constexpr int SET = 64 / EPS;         // steps of a set of 64 entries
    __shared__ float sm_m[WAVES][16], sm_l[WAVES][16];
    __shared__ __align__(16) float sm_o[WAVES][16][D + 4];

    const int u = blockIdx.x, split = blockIdx.y, splits = gridDim.y;
    const int b = u / a.Hkv, g = u - b * a.Hkv;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int L = lane >> 4, col = lane & 15;
    const int n_entries = entries_of(a, b);
    const int nsteps = (int)(((int64_t)n_entries * BLK + TOK - 1) / TOK);
    const int s_begin = split * a.steps_per_split, s_end = min(s_begin + a.steps_per_split, nsteps);
    const int open_rows = a.open ? max(a.len[b], 0) & (BLK - 1) : 0;
    const bool tail = split == 0 && open_rows > 0;
    float *part = a.ws + ((int64_t)u * splits + split) * a.G * (D + 2);
    if (s_begin >= nsteps && !tail) {  // nothing here: the merge drops it by its maximum
        if (splits > 1) {
            if (threadIdx.x < a.G) part[threadIdx.x * (D + 2)] = -INFINITY;
        } else {
            for (int i = threadIdx.x; i < a.G * D; i += blockDim.x) a.out[((int64_t)b * a.Hq + g * a.G) * D + i] = 0.f;
        }
        return;
    }

    // B operand of S^T: head `col`, channels 64*(m/2) + 16L + 8*(m%2) .. +7
    frag_t qf[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const int h = col < a.G ? col : 0;
        const u32x4_t w = *reinterpret_cast<const u32x4_t *>(a.q + ((int64_t)b * a.Hq + g * a.G + h) * D + 64 * (m >> 1) + 16 * L + 8 * (m & 1));
        qf[m].u = col < a.G ? w : u32x4_t{0, 0, 0, 0};
    }

    const gptr_t base = (gptr_t)(a.kv + a.region_off[u]);
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

    float mrun = -INFINITY, lrun = 0.f;
    f32x4_t o[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) o[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    // logits z (exp2 domain, -inf where masked) of the lane's tokens 4L + i of
    // both subtiles, V scales and operand: one online softmax step
    auto attend = [&](const float (&z)[8], float sv0, float sv1, auto &&vfrag) {
        float cm = fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
        cm = rows_max(cm);
        const float mnew = fmaxf(mrun, cm);
        const float m0 = mnew == -INFINITY ? 0.f : mnew;  // nothing yet: every p is 0
        if (__builtin_expect(__any(mnew != mrun), 0)) {
            const float alpha = __builtin_amdgcn_exp2f(mrun - m0);
#pragma unroll
            for (int t = 0; t < 8; ++t) o[t] *= alpha;
            lrun *= alpha;
            mrun = mnew;
        }
        frag_t p1, p2, p3;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            float x[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float p = __builtin_amdgcn_exp2f(z[i + h] - m0);
                lrun += p;
                x[h] = p * (i < 4 ? sv0 : sv1);
            }
            // three parts by truncation: each takes the upper half of what is left
            auto upper = [&] { return __builtin_amdgcn_perm(__float_as_uint(x[1]), __float_as_uint(x[0]), 0x07060302); };
            auto drop = [&](uint32_t w) {
                x[0] -= __uint_as_float(w << 16);
                x[1] -= __uint_as_float(w & 0xFFFF0000u);
            };
            p1.w[i >> 1] = upper();
            drop(p1.w[i >> 1]);
            p2.w[i >> 1] = upper();
            drop(p2.w[i >> 1]);
            p3.w[i >> 1] = upper();
        }
        // four accumulators in turn, so that none waits for its last product
#pragma unroll
        for (int t = 0; t < 8; t += 4) {
            frag_t v[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) v[h] = vfrag(t + h);
#pragma unroll
            for (int h = 0; h < 4; ++h) o[t + h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[h].v, p1.v, o[t + h], 0, 0, 0);
#pragma unroll
            for (int h = 0; h < 4; ++h) o[t + h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[h].v, p2.v, o[t + h], 0, 0, 0);
#pragma unroll
            for (int h = 0; h < 4; ++h) o[t + h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[h].v, p3.v, o[t + h], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
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
    auto compute_step = [&](const step_t &x) {
        float z[8];
        f32x4_t acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                frag_t f;
                widen4<FMT>(x.k[2 * s + (m >> 1)][2 * (m & 1)], f.w[0], f.w[1]);
                widen4<FMT>(x.k[2 * s + (m >> 1)][2 * (m & 1) + 1], f.w[2], f.w[3]);
                acc[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.v, qf[m].v, acc[s], 0, 0, 0);
            }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const float sk = x.sc[s].x * a.scale_log2;
#pragma unroll
            for (int i = 0; i < 4; ++i) z[4 * s + i] = x.ok[s] ? acc[s][i] * sk : -INFINITY;
        }
        attend(z, x.sc[0].y, x.sc[1].y, [&](int t) {
            frag_t f;
            widen4<FMT>(x.v[t >> 2][t & 3], f.w[0], f.w[1]);
            widen4<FMT>(x.v[2 + (t >> 2)][t & 3], f.w[2], f.w[3]);
            return f;
        });
    };

    int st = s_begin + wave;
    int pages = resolve(st), ahead = resolve(st + SET * WAVES);
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

    step_t bufA, bufB;
    load_next(bufA);

    if (tail && wave == WAVES - 1) {
        // the open record: bf16 rows of K, channel-major V, tokens past the last not read
        const uint8_t *ok = a.open + (int64_t)u * OPEN;
        const uint16_t *ov = reinterpret_cast<const uint16_t *>(ok + BLK * D * 2);
        float z[8];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                frag_t f;
                f.u = u32x4_t{0, 0, 0, 0};
                if (16 * s + col < open_rows)
                    f.u = *reinterpret_cast<const u32x4_t *>(ok + (16 * s + col) * (D * 2) + (64 * (m >> 1) + 16 * L + 8 * (m & 1)) * 2);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f.v, qf[m].v, acc, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) z[4 * s + i] = 16 * s + 4 * L + i < open_rows ? acc[i] * a.scale_log2 : -INFINITY;
        }
        attend(z, 1.f, 1.f, [&](int t) {
            frag_t f;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int tok = 16 * s + 4 * L, left = open_rows - tok;  // the lane's live tokens
                u32x2_t w = {0, 0};
                if (left > 0) w = *reinterpret_cast<const u32x2_t *>(ov + (8 * col + t) * BLK + tok);
                f.w[2 * s] = left > 1 ? w.x : w.x & 0xFFFFu;
                f.w[2 * s + 1] = left > 3 ? w.y : left > 2 ? w.y & 0xFFFFu : 0u;
            }
            return f;
        });
    }

    for (; st < s_end; st += 2 * WAVES) {
        load_next(bufB);
        compute_step(bufA);
        if (st + WAVES >= s_end) break;
        load_next(bufA);
        compute_step(bufB);
    }
    lrun += __shfl_xor(lrun, 16);
    lrun += __shfl_xor(lrun, 32);

    // wave partials -> LDS; the lane holds channels 32L + 8i + t of head `col`
    if (L == 0) {
        sm_m[wave][col] = mrun;
        sm_l[wave][col] = lrun;
    }
    if (col < a.G) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float *row = &sm_o[wave][col][32 * L + 8 * i];
            *reinterpret_cast<f32x4_t *>(row) = f32x4_t{o[0][i], o[1][i], o[2][i], o[3][i]};
            *reinterpret_cast<f32x4_t *>(row + 4) = f32x4_t{o[4][i], o[5][i], o[6][i], o[7][i]};
        }
    }
    __syncthreads();
    for (int idx = threadIdx.x; idx < a.G * D; idx += WAVES * 64) {
        const int h = idx / D, ch = idx - h * D;
        float M = sm_m[0][h];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) M = fmaxf(M, sm_m[w][h]);
        const float m0 = M == -INFINITY ? 0.f : M;
        float lsum = 0.f, osum = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float sc = __builtin_amdgcn_exp2f(sm_m[w][h] - m0);
            lsum += sc * sm_l[w][h];
            osum += sc * sm_o[w][h][ch];
        }
        if (splits == 1) {
            a.out[((int64_t)b * a.Hq + g * a.G) * D + idx] = lsum == 0.f ? 0.f : osum / lsum;
        } else {
            float *pp = part + h * (D + 2);
            if (ch == 0) {
                // a split that saw only NaN logits is kept: its sums are NaN
                pp[0] = M == -INFINITY && lsum != 0.f ? 0.f : M;
                pp[1] = lsum;
            }
            pp[2 + ch] = osum;
        }
    }
}

// Merges a unit's splits in their order, one workgroup per (unit, head), two
// channels a lane.  Each of the W waves takes up to N splits, whose partials
// it reads at once, beside all splits' maxima and sums (a split a lane): no
// load waits for another.  A split without a token has the maximum -inf and
// no partial.
template <int W, int N>
__global__ __launch_bounds__(W * 64) void combine_kv8_kernel(const float *__restrict__ ws, int Hq, int Hkv, int G,
                                                             int splits, float *__restrict__ out)
{
    constexpr int PER = (W * N + 63) / 64;  // splits of a lane
    typedef float f2_t __attribute__((ext_vector_type(2), aligned(4)));
    __shared__ f32x2_t s_o[W][64];
    const int u = blockIdx.x, h = blockIdx.y, lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t stride = (int64_t)G * (D + 2);
    const float *p = ws + (int64_t)u * splits * stride + h * (D + 2);
    f2_t x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = *reinterpret_cast<const f2_t *>(p + min(wave * N + i, splits - 1) * stride + 2 + 2 * lane);
    f2_t ml[PER];
    float M = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        ml[i] = f2_t{-INFINITY, 0.f};
        if (i * 64 + lane < splits) ml[i] = *reinterpret_cast<const f2_t *>(p + (i * 64 + lane) * stride);
        M = fmaxf(M, ml[i].x);
    }
    M = wave_max(M);
    const float m0 = M == -INFINITY ? 0.f : M;
    float w[PER], lsum = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        w[i] = __builtin_amdgcn_exp2f(ml[i].x - m0);
        lsum += ml[i].x == -INFINITY ? 0.f : w[i] * ml[i].y;
    }
    f32x2_t osum = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int s = wave * N + i;  // its weight: lane s % 64 of the s / 64-th
        float own = w[0];
#pragma unroll
        for (int j = 1; j < PER; ++j) own = s / 64 == j ? w[j] : own;
        const float sc = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(own), s % 64));
        if (s < splits && sc != 0.f) {
            osum.x += sc * x[i].x;
            osum.y += sc * x[i].y;
        }
    }
    if (wave) s_o[wave][lane] = osum;
    if (W > 1) __syncthreads();
    if (wave) return;
#pragma unroll
    for (int j = 1; j < W; ++j) {
        osum.x += s_o[j][lane].x;
        osum.y += s_o[j][lane].y;
    }
    lsum = wave_sum(lsum);
    f2_t y = {0.f, 0.f};
    if (lsum != 0.f) y = f2_t{osum.x / lsum, osum.y / lsum};
    const int b = u / Hkv, g = u - b * Hkv;
    *reinterpret_cast<f2_t *>(out + ((int64_t)b * Hq + g * G + h) * D + 2 * lane) = y;
}

struct split_plan {
    int splits, steps_per_split;
};

// Splits per unit: three workgroups a CU, 8 steps or more each.
split_plan plan(int64_t units, int k, int blk, int most)
{
    const int steps = (int)(((int64_t)k * blk + TOK - 1) / TOK);
    int64_t n = std::min<int64_t>((3 * CUS + units - 1) / units, std::max(1, steps / 8));
    n = std::min<int64_t>(n, std::min<int64_t>(most, kMaxPartials / std::max<int64_t>(units, 1)));
    n = std::max<int64_t>(n, 1);
    const int per = (int)((steps + n - 1) / n);
    return {(steps + per - 1) / per, per};
}

bool has_plan(int B, int Hq, int Hkv, int d, int blk, int k)
{
    return B > 0 && Hkv > 0 && Hq > 0 && Hq % Hkv == 0 && d == D && ss::supported_blk(blk) && k > 0;
}

size_t split_bytes(int B, int Hq) { return (size_t)B * Hq * (D + 2) * sizeof(float); }

template <int FMT>
auto attn_of(int blk)
{
    return blk == 8 ? attn_kv8_kernel<8, FMT> : blk == 16 ? attn_kv8_kernel<16, FMT> : attn_kv8_kernel<32, FMT>;
}

}  // namespace

extern "C" size_t ss_sparse_attention_kv8_workspace(int B, int Hq, int Hkv, int d, int blk, int k)
{
    if (!has_plan(B, Hq, Hkv, d, blk, k)) return 0;
    const int splits = plan((int64_t)B * Hkv, k, blk, kMaxSplits).splits;
    return splits > 1 ? splits * split_bytes(B, Hq) : 0;
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
    SS_CHECK_SUPPORTED(units <= 0x7FFFFFFF / (WAVES * 64), "ss_sparse_attention_kv8: %lld units pass the launch", (long long)units);
    const size_t room = workspace ? ws_bytes / split_bytes(B, Hq) : 0;
    const split_plan sp = plan(units, k, blk, (int)std::max<size_t>(1, std::min(room, (size_t)kMaxSplits)));
    const int G = Hq / Hkv;
    const attn_args a = {static_cast<const uint16_t *>(q), static_cast<const uint8_t *>(kv_base), region_off, sel, tables,
                         max_blocks, capacity, slot_limit, nblk, static_cast<const uint8_t *>(open_blocks), len, Hq, Hkv, G,
                         k, scale * 1.4426950408889634f, sp.steps_per_split, out, static_cast<float *>(workspace)};
    hipStream_t s = ss::as_stream(stream);
    ss::launch(fmt == SS_KV8_E4M3 ? attn_of<SS_KV8_E4M3>(blk) : attn_of<SS_KV8_INT8>(blk), dim3((unsigned)units, sp.splits),
               dim3(WAVES * 64), s, a);
    ss_status st = ss::check_launch("ss_sparse_attention_kv8");
    if (st != SS_OK || sp.splits == 1) return st;
    // reads as many partials as there may be splits
    auto *combine = combine_kv8_kernel<16, 16>;
    int waves = 16;
    if (sp.splits <= 4) combine = combine_kv8_kernel<1, 4>, waves = 1;
    else if (sp.splits <= 8) combine = combine_kv8_kernel<1, 8>, waves = 1;
    else if (sp.splits <= 16) combine = combine_kv8_kernel<2, 8>, waves = 2;
    else if (sp.splits <= 32) combine = combine_kv8_kernel<4, 8>, waves = 4;
    else if (sp.splits <= 64) combine = combine_kv8_kernel<8, 8>, waves = 8;
    else if (sp.splits <= 128) combine = combine_kv8_kernel<16, 8>, waves = 16;
    combine<<<dim3((unsigned)units, G), dim3(waves * 64), 0, s>>>(a.ws, Hq, Hkv, G, sp.splits, out);
    return ss::check_launch("ss_sparse_attention_kv8(merge)");
}
