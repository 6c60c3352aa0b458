// Gradients of the attention over another sequence's states.
//
// With P = exp(scale * Q K^T - lse), dP = dO V^T and D_i = sum_j P_ij dP_ij (which is sum_c dO_ic O_ic):
//     dS = P o (dP - D)     dV = P^T dO     dK = scale * dS^T Q     dQ = scale * dS K
// Nothing of size M x N meets memory.  Two passes, each of which owns what it sums, so that nothing is added atomically and a result does not depend on
// timing: one over rows (a workgroup keeps its queries and walks the keys: dQ, D), one over keys (keeps its keys and walks the queries: dK, dV).
// S and dP are computed in both: 8 products instead of 5.  Both compute the transposes of S and dP resp. S and dP themselves such that a lane owns one row
// (one key), as in the forward pass: probabilities and dS come out of the first products in the layout in which the last ones read them.
//
// D.  O was rounded to 16 bits, and dO . O is off by that times |O|, however little dP - D is beside it (values of 8 and a tenth around it, bf16: dQ off by 0.16 of itself).  The pass over rows
// therefore takes D' = dO . O for a first estimate only.  Over its walk it sums e = sum_j P (dP - D') = D - D', and P K beside dS' K, whose operands are the same:
//     D = D' + e     dQ = scale * (sum_j dS'_ij K_j - e * sum_j P_ij K_j)
// and the pass over keys reads that D.  What the roundings of P and dS' leave of the estimate's error is u^2 |dO| |O|, beside dS' own u |dS| (u: the input type's half step).
//
// LDS tiles [rows][128 bytes] per 64 channels are read both along their rows (S, dP) and across them (dQ, dK, dV: the transposing read).
// 16-byte column c of row r is kept at column c ^ (4 * (r/2 mod 2) + r/4 mod 4): the 16 rows of a ds_read_b128 phase meet all banks once, and the 8 rows
// whose 64-byte segments one transposing read takes lie in both halves of a 128-byte row, the least a 512-byte read can do.
//
// Roundings: P and dS are rounded to the input type for the last products (in small calls in two parts, see kTwoParts).  BF16 has fp32's range.  In F16 a probability is held times 2^14, and dS times a power
// of two per row (per key) that keeps the largest so far below 2^15: gradients arrive at any magnitude, and dS relative to 1 would fall among F16's subnormals where dQ does not.
#pragma once
#include "tir_kernel.h"

namespace tir {

struct GradParams {
    const void *Q, *K, *V, *O, *dO;
    void *dQ, *dK, *dV;
    const float* lse;        // [batch][query heads][M]
    float* delta;            // the same: D, written by the pass over rows (its slices' sum)
    const int* lens;         // null: N each
    long long q_bs, q_rs, q_hs, k_bs, k_rs, k_hs, v_bs, v_rs, v_hs, o_bs, o_rs, o_hs, g_bs, g_rs, g_hs;      // (g: dO)
    int q_near;              // 128 positions and all heads of a group lie within 2^31 bytes of dQ
    int M, N, heads, G;      // key heads, query heads per key head
    int batch, tiles;        // tiles of rows resp. keys of a (sequence, key head)
    int slices;              // workgroups that share a tile's walk: partial sums in ws, added by grad_sum_kernel
    float scale, scale_log2e;
    float* ws;
    unsigned div_h_magic, div_g_magic, div_tiles_magic;
    int div_h_shift, div_g_shift, div_tiles_shift;
};

constexpr int kGradWaves = 4, kGradThreads = 64 * kGradWaves, kGradTile = 32 * kGradWaves;      // rows resp. keys of a workgroup
// Pairs (query, key) of a call, all heads together, up to which P and dS are operands in two parts: a value rounded to 16 bits and what that left of it, rounded likewise.  One rounding of a
// probability is up to u of a sum that it dominates, and as much again as the result's own rounding in the mean; over many they even out to 1.42 of it, over a few hundred they may reach 1.6 (2 x 110 keys x
// 8 heads of 128, bf16: dV off by 2.6e-3, 1.66e-3 in two parts).  Calls this small mostly wait for memory and launches: that one takes 17.2 us instead of 16.1, 27 x 2 keys x 2 x 3 heads 12.6 instead of 12.0, one token x 500 keys x
// 8 heads on one 24.5 instead of 22.7, 128 x 128 keys 21.2 instead of 19.1, 16 x 1 x 64 keys x 16 heads of 64 12.4 instead of 11.8.  Only where the pass over keys takes two row groups: the other form has no registers left at d = 64.
constexpr int kTwoParts = 1 << 14;
constexpr int kFewKeys = 64;        // up to so many keys are one chunk of the pass over rows

// Partial sums of a slice, in floats.  Rows: dS' K, P K and the rows' e; keys: dK and dV.
constexpr int grad_partial(bool keys, int d) { return 2 * kGradTile * d + (keys ? 0 : kGradTile); }

hipError_t launch_grad_rows(const GradParams& p, int dt, int dh, bool two, hipStream_t stream);      // (two: operands in two parts)
hipError_t launch_grad_keys(const GradParams& p, int dt, int dh, bool two, hipStream_t stream);

__device__ __forceinline__ int grad_swz(int row) { return ((row & 2) << 1) | ((row >> 2) & 3); }

// One wave's part of a workgroup's copy of RB rows of DH channels into an LDS tile.
template <int DH, int RB> struct GradTile {
    static constexpr int HALVES = DH / 64, HALF = RB * 128, BYTES = HALVES * HALF, ROW = DH * 2;
    static constexpr int PASSES = RB / (8 * kGradWaves);      // of 8 rows per wave and half
    static_assert(PASSES >= 1, "");
    static __device__ __forceinline__ unsigned lane_offset(int wave, int lane, int rs) {      // (rs in elements)
        const int row = wave * 8 + (lane >> 3);
        return (unsigned)(row * rs * 2 + (((lane & 7) ^ grad_swz(row)) << 4));
    }
    // (rows from `left` on are zeros, whatever the stride: where it is less than a row, they would lie before the descriptor's end)
    static __device__ __forceinline__ void copy(char* tile, const char* base, int left, int rs, unsigned off, int wave, int lane) {
        const int rows = left < RB ? left : RB, row = wave * 8 + (lane >> 3);
        const i32x4 r = make_rsrc32(base, rows > 0 ? (unsigned)((rows - 1) * rs * 2 + ROW) : 0u);      // (rs of at most 2^23)
#pragma unroll
        for (int u = 0; u < PASSES; ++u) {
            const unsigned at = row + u * kGradWaves * 8 < left ? off : kOutOfRange;
#pragma unroll
            for (int h = 0; h < HALVES; ++h) load_to_lds_at(r, tile + h * HALF + (u * kGradWaves + wave) * 1024, at, u * kGradWaves * 8 * rs * 2 + h * 128);
        }
    }
    // Operand of k-step ks (16 channels): row l31 of the 32 from row r0
    static __device__ __forceinline__ const char* along_at(const char* tile, int r0, int ks, int l31, int g) {
        return tile + (ks >> 2) * HALF + (r0 + l31) * 128 + ((((ks & 3) * 2 + g) ^ grad_swz(l31)) << 4);
    }
    static __device__ __forceinline__ uint4 along(const char* tile, int r0, int ks, int l31, int g) { return *(const uint4*)along_at(tile, r0, ks, l31, g); }
    // Operand of the 16 rows from r0 for channels 32*db ..: position (g, 4*hh + e) is row r0 + 8*hh + 4*g + e, the order of a product's result registers
    static __device__ __forceinline__ uint4 across(const char* tile, int r0, int db, int blk, int s16) {
        i16x4 h[2];
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
            const int row = hh * 8 + 4 * (blk >> 1) + (s16 >> 2);
            const int col = (db & 1) * 4 + 2 * (blk & 1) + ((s16 & 3) >> 1);
            const char* const ptr = tile + (db >> 1) * HALF + (r0 + row) * 128 + ((col ^ grad_swz(row)) << 4) + (s16 & 1) * 8;
            h[hh] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(TIR_LDS_PTR(i16x4, ptr));
        }
        const i32x2 lo = __builtin_bit_cast(i32x2, h[0]), hi = __builtin_bit_cast(i32x2, h[1]);
        return make_uint4((unsigned)lo[0], (unsigned)lo[1], (unsigned)hi[0], (unsigned)hi[1]);
    }
};

// 64 consecutive floats from a descriptor into LDS, one per lane.
__device__ __forceinline__ void floats_to_lds(const i32x4& rsrc, const char* lds_base, unsigned voffset) {
    const unsigned lds_addr = (unsigned)(unsigned long long)TIR_LDS_PTR(const char, lds_base);
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 0\n\t"
        "buffer_load_dword %1, %2, 0 offen lds"
        :
        : "s"(lds_addr), "v"(voffset), "s"(rsrc)
        : "memory", "m0");
}

template <int DT> __device__ __forceinline__ unsigned grad_pack(float a, float b) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    if constexpr (DT == DT_F16) {
        const h2 v = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(unsigned, v);
    } else {
        const b2 v = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(unsigned, v);
    }
}
// Sum of the products of two operands' eight values.
template <int DT> __device__ __forceinline__ float dot8(const uint4& a, const uint4& b) {
    const unsigned x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float u[2], v[2];
        if constexpr (DT == DT_F16) {
            typedef _Float16 h2 __attribute__((ext_vector_type(2)));
            const h2 p = __builtin_bit_cast(h2, x[i]), q = __builtin_bit_cast(h2, y[i]);
            u[0] = (float)p[0]; u[1] = (float)p[1];
            v[0] = (float)q[0]; v[1] = (float)q[1];
        } else {
            u[0] = __builtin_bit_cast(float, x[i] << 16); u[1] = __builtin_bit_cast(float, x[i] & 0xffff0000u);
            v[0] = __builtin_bit_cast(float, y[i] << 16); v[1] = __builtin_bit_cast(float, y[i] & 0xffff0000u);
        }
        s = __builtin_fmaf(u[0], v[0], s);
        s = __builtin_fmaf(u[1], v[1], s);
    }
    return s;
}
__device__ __forceinline__ float grad_half_max(float x) {      // over the two half-waves
    const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    const unsigned lo = both[0], hi = both[1];
    return __builtin_fmaxf(__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi));
}

// dS of 32 x 32 pairs, rounded for the last product.  `by`: the power of two that a lane's row (key) is held times; where it shrinks, so do the sums in acc.
template <int DT, int DB> __device__ __forceinline__ void round_ds(f32x16& ds, float& by, f32x16 (&acc)[DB], unsigned (&w)[8]) {
    if constexpr (DT == DT_F16) {
        float top = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) top = __builtin_fmaxf(top, __builtin_fabsf(ds[r]));
        top = grad_half_max(top);
        if (__builtin_amdgcn_ballot_w64(top * by >= 0x1p15f) != 0) {
            // 2^(14 - e) with top < 2^e: below 2^14, and room for twice as much to come (an infinite or NaN dS: the factor stays, the result shows it)
            const float fresh = __builtin_amdgcn_ldexpf(1.f, 14 - __builtin_amdgcn_frexp_expf(top));
            const float next = top * by >= 0x1p15f && top < __builtin_inff() ? fresh : by;
            const float f = next / by;
            by = next;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[db][r] *= f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = grad_pack<DT>(ds[2 * i] * by, ds[2 * i + 1] * by);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = grad_pack<DT>(ds[2 * i], ds[2 * i + 1]);
    }
}
// What the rounding of x * by to w left of it, rounded likewise: a second operand.
template <int DT> __device__ __forceinline__ void rest_of(const f32x16& x, float by, unsigned (&w)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float lo, hi;
        if constexpr (DT == DT_F16) {
            typedef _Float16 h2 __attribute__((ext_vector_type(2)));
            const h2 v = __builtin_bit_cast(h2, w[i]);
            lo = (float)v[0];
            hi = (float)v[1];
        } else {
            lo = __builtin_bit_cast(float, w[i] << 16);
            hi = __builtin_bit_cast(float, w[i] & 0xffff0000u);
        }
        w[i] = grad_pack<DT>(__builtin_fmaf(x[2 * i], by, -lo), __builtin_fmaf(x[2 * i + 1], by, -hi));
    }
}
// Four values of a row into a tile of rows in LDS, and that tile to memory in 16-byte pieces: a row's values lie in two lanes, 8 bytes at a time.  Written through (see the forward kernels);
// `near`: the tile's rows lie within 2^31 bytes.  place(r): elements from base to row r.  Threads of the workgroup (T = its size) or of a wave (64) take part.
template <int DH> __device__ __forceinline__ void grad_stage(char* tile, int row, int ch, uint2 v) { *(uint2*)(tile + row * (DH * 2) + ((ch * 2) ^ ((row & 7) << 4))) = v; }
template <int DH, int T, class PLACE> __device__ __forceinline__ void grad_store(const char* tile, unsigned short* base, int rows, bool near, PLACE place) {
    typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
    constexpr int RC = DH / 8, ROWS = T == 64 ? 32 : kGradTile;      // 16-byte pieces of a row
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, 0x7fffffff, 0x00020000);
#pragma unroll
    for (int i = 0; i < ROWS * RC / T; ++i) {
        const int q = (int)(threadIdx.x & (T - 1)) + i * T, row = q / RC, pc = q % RC;
        const u32x4 v = *(const u32x4*)(tile + row * (DH * 2) + ((pc * 16) ^ ((row & 7) << 4)));
        const long long at = place(row) + pc * 8;
        if (near) __builtin_amdgcn_raw_buffer_store_b128(v, r, row < rows ? (int)at * 2 : (int)kOutOfRange, 0, TIR_STORE_AUX);
        else if (row < rows) *(u32x4*)(base + at) = v;
    }
}
constexpr float kFirstFactor = 0x1p100f;      // before any dS has been seen
template <int DT> __device__ __forceinline__ float p_factor_log2() { return DT == DT_F16 ? 14.f : 0.f; }

// The values are there at this point of the program: products are not moved behind what follows, where more of their operands would be held at a time.
__device__ __forceinline__ void here(f32x16& x) { asm volatile("" : "+v"(x)); }

struct TwoOperands {
    uint4 a, b;
};
// N products with their operands read from LDS LA products ahead; nothing else moves between them, so that no more than LA operands are held.
template <int N, int LA, class READ, class MUL> __device__ __forceinline__ void products(READ read, MUL mul) {
    decltype(read(0)) f[LA];
#pragma unroll
    for (int t = 0; t < LA; ++t) f[t] = read(t);
    TIR_FENCE();
#pragma unroll
    for (int t = 0; t < N; ++t) {
        mul(t, f[t % LA]);
        TIR_FENCE();
        if (t + LA < N) f[t % LA] = read(t + LA);
        TIR_FENCE();
    }
}

// ---------------------------------------------------------------------------------------------
// dQ and D: four waves of 32 rows (position, query head) each; keys and values through two LDS stages.
//
// FEW: calls of up to kFewKeys keys.  All terms of D are at hand before the first dS is formed, so it is summed from them and neither O nor P K is needed
// (3 x 2500 x 19 keys x 56 query heads of 128: 172 us when O was read, 144 without).
// Otherwise, at d = 128, the two sums are 128 registers and the queries 32; dO is kept in LDS, beside chunks of half as many keys.  The second sum costs a third of the matrix work and half of
// the vector registers: both passes with and without it, 2 x 2047 x 4095 and 1365 keys x 16 / 4 heads of 128 400 and 353 us, 16 x 250 x 333 x 12 heads of 64 33.4 and 31.9 (two workgroups per CU and three).
// ---------------------------------------------------------------------------------------------
template <int DT, int DH, bool FEW, bool TWO>
__global__ void __launch_bounds__(kGradThreads, 2) grad_rows_kernel(const GradParams p) {
    constexpr int CH = FEW || DH == 64 ? 64 : 32;      // keys of a chunk
    constexpr bool G_LDS = !FEW && DH == 128;
    constexpr int LA = 2;
    static_assert(!FEW || CH == kFewKeys, "");
    typedef GradTile<DH, CH> T;
    typedef GradTile<DH, kGradTile> GT;
    constexpr int KSTEPS = DH / 16, DB = DH / 32, STAGE = 2 * T::BYTES, RING = (FEW ? 1 : 2) * STAGE;
    static_assert(RING >= kGradTile * DH * 2, "the output tile is staged in the ring");
    __shared__ __attribute__((aligned(1024))) char smem[RING + (G_LDS ? GT::BYTES : 0)];
    const int lane = threadIdx.x & 63, l31 = lane & 31, g = lane >> 5, blk = lane >> 4, s16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int bh = (int)fastdiv(blockIdx.x, p.div_tiles_magic, p.div_tiles_shift);
    const int row0 = ((int)blockIdx.x - bh * p.tiles) * kGradTile;
    const int b = (int)fastdiv((unsigned)bh, p.div_h_magic, p.div_h_shift), h = bh - b * p.heads;
    const int rows = p.M * p.G - row0 < kGradTile ? p.M * p.G - row0 : kGradTile;
    int n = p.N;
    if (p.lens) {
        n = p.lens[b];
        n = n < 0 ? 0 : (n > p.N ? p.N : n);
    }
    const int chunks_all = (n + CH - 1) / CH;
    const int per = FEW ? chunks_all : (chunks_all + p.slices - 1) / p.slices;
    const int c0 = FEW ? 0 : (int)blockIdx.y * per;
    const int chunks = chunks_all - c0 < per ? chunks_all - c0 : per;      // may be none: this slice's sums are zeros

    const char* const Kb = (const char*)p.K + 2 * (b * p.k_bs + h * p.k_hs);
    const char* const Vb = (const char*)p.V + 2 * (b * p.v_bs + h * p.v_hs);
    const int k_rs = (int)p.k_rs, v_rs = (int)p.v_rs;
    const unsigned k_off = T::lane_offset(wave, lane, k_rs), v_off = T::lane_offset(wave, lane, v_rs);
    auto copy = [&](int i) __attribute__((always_inline)) {
        char* const st = smem + (FEW ? 0 : (i & 1) * STAGE);
        const long long key = (long long)(c0 + i) * CH;
        const int left = i < chunks ? n - (int)key : 0;
        T::copy(st, Kb + key * k_rs * 2, left, k_rs, k_off, wave, lane);
        T::copy(st + T::BYTES, Vb + key * v_rs * 2, left, v_rs, v_off, wave, lane);
    };
    if (chunks > 0) copy(0);

    // this lane's row
    const int row = row0 + wave * 32 + l31;
    const bool live = wave * 32 + l31 < rows;
    const int m = (int)fastdiv((unsigned)row, p.div_g_magic, p.div_g_shift), hq = h * p.G + row - m * p.G;
    uint4 qf[KSTEPS], of[G_LDS ? 1 : KSTEPS];
    float delta = 0.f, lse2 = 0.f;
    const long long stat = ((long long)b * p.heads * p.G + hq) * p.M + m;
    char* const g_tile = smem + RING;                  // G_LDS: a wave writes and reads its own 32 rows
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) qf[ks] = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int ks = 0; ks < (G_LDS ? 1 : KSTEPS); ++ks) of[ks] = make_uint4(0, 0, 0, 0);
    {
        const char* const q = (const char*)p.Q + 2 * (b * p.q_bs + m * p.q_rs + hq * p.q_hs) + g * 16;
        const char* const go = (const char*)p.dO + 2 * (b * p.g_bs + m * p.g_rs + hq * p.g_hs) + g * 16;
        const char* const o = (const char*)p.O + 2 * (b * p.o_bs + m * p.o_rs + hq * p.o_hs) + g * 16;
        if constexpr (G_LDS) {
            uint4 x[KSTEPS];
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks) x[ks] = make_uint4(0, 0, 0, 0);
            if (live) {
#pragma unroll
                for (int ks = 0; ks < KSTEPS; ++ks) {
                    x[ks] = *(const uint4*)(go + ks * 32);
                    delta += dot8<DT>(x[ks], *(const uint4*)(o + ks * 32));
                }
            }
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks) *(uint4*)(g_tile + (GT::along_at(g_tile, wave * 32, ks, l31, g) - g_tile)) = x[ks];
            TIR_FENCE();
        }
        if (live) {
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks) {
                qf[ks] = *(const uint4*)(q + ks * 32);
                if constexpr (!G_LDS) of[ks] = *(const uint4*)(go + ks * 32);
                if constexpr (!G_LDS && !FEW) delta += dot8<DT>(of[ks], *(const uint4*)(o + ks * 32));
            }
            lse2 = p.lse[stat] * 1.44269504088896340736f;
        }
    }
    const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    float first = 0.f;                                 // dP of the row's first key: D is summed from it on, and a single key's D is its dP to the bit, as its dS of zero has to be
    if (FEW && chunks > 0) {
        copy_barrier<0>();
#pragma unroll 1
        for (int jb = 0; jb * 32 < n; ++jb) {
            f32x16 s, dp;
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks) s = InTraits<DT>::mfma(T::along(smem, jb * 32, ks, l31, g), qf[ks], ks == 0 ? zero16 : s);
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks) dp = InTraits<DT>::mfma(T::along(smem + T::BYTES, jb * 32, ks, l31, g), of[ks], ks == 0 ? zero16 : dp);
            if (jb == 0) first = __shfl(dp[0], l31);
#pragma unroll
            for (int r = 0; r < 16; ++r) delta += jb * 32 + 8 * (r >> 2) + 4 * g + (r & 3) < n ? __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], p.scale_log2e, -lse2)) * (dp[r] - first) : 0.f;
        }
    }
    delta += __shfl_xor(delta, 32);
    if (FEW) delta += first;

    f32x16 acc[DB], pk[FEW ? 1 : DB];                  // sums of dS' K and of P K
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] = pk[FEW ? 0 : db][r] = 0.f;
    float by = DT == DT_F16 ? kFirstFactor : 1.f, e_sum = 0.f;
    const float ref2 = FEW ? -lse2 : p_factor_log2<DT>() - lse2, pf = FEW || DT != DT_F16 ? 1.f : 0x1p-14f;      // (a probability that is an operand is held times 2^14 in F16)

    for (int i = 0; i < chunks; ++i) {
        copy_barrier<0>();                     // chunk i is in, and everybody is past chunk i - 1
        if (i + 1 < chunks) copy(i + 1);
        const char* const tk = smem + (FEW ? 0 : (i & 1) * STAGE);
        const char* const tv = tk + T::BYTES;
#pragma unroll
        for (int jb = 0; jb < CH / 32; ++jb) {
            const int left = n - (c0 + i) * CH - jb * 32;      // keys of this block
            if (left <= 0) break;
            f32x16 s, dp;
            unsigned w[8], pw[8];
            if constexpr (FEW) {
#pragma unroll
                for (int ks = 0; ks < KSTEPS; ++ks) s = InTraits<DT>::mfma(T::along(tk, jb * 32, ks, l31, g), qf[ks], ks == 0 ? zero16 : s);
#pragma unroll
                for (int ks = 0; ks < KSTEPS; ++ks) dp = InTraits<DT>::mfma(T::along(tv, jb * 32, ks, l31, g), of[ks], ks == 0 ? zero16 : dp);
            } else {
                products<KSTEPS, LA>([&](int ks) __attribute__((always_inline)) { return T::along(tk, jb * 32, ks, l31, g); },
                                     [&](int ks, const uint4& x) __attribute__((always_inline)) { s = InTraits<DT>::mfma(x, qf[ks], ks == 0 ? zero16 : s); });
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], p.scale_log2e, ref2));
            if (left < 32) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + 4 * g + (r & 3) < left ? s[r] : 0.f;
            }
            if constexpr (G_LDS)
                products<KSTEPS, LA>([&](int ks) __attribute__((always_inline)) { return TwoOperands{T::along(tv, jb * 32, ks, l31, g), GT::along(g_tile, wave * 32, ks, l31, g)}; },
                                     [&](int ks, const TwoOperands& x) __attribute__((always_inline)) { dp = InTraits<DT>::mfma(x.a, x.b, ks == 0 ? zero16 : dp); });
            else if constexpr (!FEW)
                products<KSTEPS, LA>([&](int ks) __attribute__((always_inline)) { return T::along(tv, jb * 32, ks, l31, g); },
                                     [&](int ks, const uint4& x) __attribute__((always_inline)) { dp = InTraits<DT>::mfma(x, of[ks], ks == 0 ? zero16 : dp); });
            f32x16 ds;
#pragma unroll
            for (int r = 0; r < 16; ++r) ds[r] = s[r] * (dp[r] - delta);
            if constexpr (FEW) {
                round_ds<DT, DB>(ds, by, acc, w);
#pragma unroll
                for (int ss = 0; ss < 2; ++ss) {
                    const uint4 df = make_uint4(w[4 * ss], w[4 * ss + 1], w[4 * ss + 2], w[4 * ss + 3]);
#pragma unroll
                    for (int db = 0; db < DB; ++db) acc[db] = InTraits<DT>::mfma(T::across(tk, jb * 32 + ss * 16, db, blk, s16), df, acc[db]);
                }
            } else {
#pragma unroll
                for (int r = 0; r < 8; ++r) pw[r] = grad_pack<DT>(s[2 * r], s[2 * r + 1]);
#pragma unroll
                for (int r = 0; r < 16; ++r) e_sum += ds[r];
                round_ds<DT, DB>(ds, by, acc, w);
                products<2 * DB, LA>([&](int t) __attribute__((always_inline)) { return T::across(tk, jb * 32 + t / DB * 16, t % DB, blk, s16); },
                                     [&](int t, const uint4& x) __attribute__((always_inline)) {
                                         const int at = t / DB * 4;
                                         acc[t % DB] = InTraits<DT>::mfma(x, make_uint4(w[at], w[at + 1], w[at + 2], w[at + 3]), acc[t % DB]);
                                         pk[t % DB] = InTraits<DT>::mfma(x, make_uint4(pw[at], pw[at + 1], pw[at + 2], pw[at + 3]), pk[t % DB]);
                                     });
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    here(acc[db]);
                    here(pk[db]);
                }
            }
            if constexpr (TWO) {
                rest_of<DT>(ds, by, w);
                products<2 * DB, LA>([&](int t) __attribute__((always_inline)) { return T::across(tk, jb * 32 + t / DB * 16, t % DB, blk, s16); },
                                     [&](int t, const uint4& x) __attribute__((always_inline)) {
                                         const int at = t / DB * 4;
                                         acc[t % DB] = InTraits<DT>::mfma(x, make_uint4(w[at], w[at + 1], w[at + 2], w[at + 3]), acc[t % DB]);
                                     });
#pragma unroll
                for (int db = 0; db < DB; ++db) here(acc[db]);
            }
            TIR_FENCE();                       // (the next block's operands read ahead of here would not fit the registers)
        }
    }
    const float f = !FEW && n == 1 ? 0.f : p.scale * pf / by;      // (a single key's dS is zero, which the rounding of an estimate would not leave)
    e_sum = (e_sum + __shfl_xor(e_sum, 32)) * pf;
    const bool whole = FEW || p.slices == 1;
    if (live && g == 0 && (whole || blockIdx.y == 0)) {
        // (the row's place once more: held over the loop, its registers would be short there)
        int r = row0 + wave * 32 + l31;
        asm volatile("" : "+v"(r));
        const int mr = (int)fastdiv((unsigned)r, p.div_g_magic, p.div_g_shift);
        p.delta[((long long)b * p.heads * p.G + h * p.G + r - mr * p.G) * p.M + mr] = whole ? delta + e_sum : delta;
    }
    const float fp = !FEW && n == 1 ? 0.f : -(p.scale * pf) * e_sum;
    if constexpr (!FEW) {
        if (p.slices > 1) {
            if (wave * 32 >= rows) return;               // (nobody reads these)
            // [tile][slice]: dS' K and P K, [wave][db][quarter][lane] of four values each, and e of the rows
            typedef float f32x4 __attribute__((ext_vector_type(4)));
            float* const part = p.ws + ((long long)blockIdx.x * p.slices + blockIdx.y) * grad_partial(false, DH);
            f32x4* const o = (f32x4*)part + wave * (32 * DH / 4) + lane;
            const float fk = n == 1 ? 0.f : p.scale * pf;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    o[(db * 4 + q4) * 64] = f32x4{acc[db][4 * q4] * f, acc[db][4 * q4 + 1] * f, acc[db][4 * q4 + 2] * f, acc[db][4 * q4 + 3] * f};
                    o[(db * 4 + q4) * 64 + kGradTile * DH / 4] = f32x4{pk[db][4 * q4] * fk, pk[db][4 * q4 + 1] * fk, pk[db][4 * q4 + 2] * fk, pk[db][4 * q4 + 3] * fk};
                }
            if (g == 0) part[2 * kGradTile * DH + wave * 32 + l31] = e_sum;
            return;
        }
    }
    __syncthreads();                           // the ring is free
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = FEW ? acc[db][4 * q4 + e] * f : __builtin_fmaf(pk[FEW ? 0 : db][4 * q4 + e], fp, acc[db][4 * q4 + e] * f);
            grad_stage<DH>(smem, wave * 32 + l31, db * 32 + q4 * 8 + 4 * g, make_uint2(grad_pack<DT>(v[0], v[1]), grad_pack<DT>(v[2], v[3])));
        }
    __syncthreads();
    const int first_m = (int)fastdiv((unsigned)row0, p.div_g_magic, p.div_g_shift);
    unsigned short* const base = (unsigned short*)p.dQ + b * p.q_bs + (long long)h * p.G * p.q_hs + first_m * p.q_rs;
    grad_store<DH, kGradThreads>(smem, base, rows, p.q_near != 0, [&](int r) __attribute__((always_inline)) -> long long {
        const int mr = (int)fastdiv((unsigned)(row0 + r), p.div_g_magic, p.div_g_shift);
        return (mr - first_m) * p.q_rs + (row0 + r - mr * p.G) * p.q_hs;
    });
}

// ---------------------------------------------------------------------------------------------
// dK and dV: four waves of 32 keys each; queries and dO, head after head, through two LDS stages with their lse and D.
//
// RG = 2: two groups of four waves on the same keys, which take every other chunk of rows through a ring each and are added through LDS at the end: two waves per SIMD where there is
// one workgroup per CU.
// A block's phases run one after the other (S and P, dV, dP and dS, dK): at d = 128 sums and keys are 160 registers, and 256 hold two waves per SIMD.  The values would be 32 more: there
// they stay in LDS, and so they do at d = 64 with RG = 1, where 168 registers then hold three workgroups per CU instead of two: 16 x 250 x 333 x 12 heads (576 workgroups) both passes 41.0 -> 37.3 us,
// 4 x 4096 x 577 x 8 heads 119 -> 114.
// ---------------------------------------------------------------------------------------------
template <int DT, int DH, int RG, bool TWO>
__global__ void __launch_bounds__(kGradThreads * RG, DH == 64 && RG == 1 ? 3 : 2) grad_keys_kernel(const GradParams p) {
    constexpr int RB = DH == 64 ? 64 : 32;              // rows of a chunk
    typedef GradTile<DH, RB> T;
    constexpr int KSTEPS = DH / 16, DB = DH / 32, STAGE = 2 * T::BYTES + 2 * RB * 4, MERGE = 2 * DB * 4096;      // (MERGE: a wave's sums)
    constexpr int LA = DH == 64 && RG == 1 ? 2 : 3;
    constexpr bool V_LDS = DH == 128 || RG == 1;
    typedef GradTile<DH, kGradTile> VT;
    constexpr int V_AT = RG * 2 * STAGE, USED = V_AT + (V_LDS ? VT::BYTES : 0);
    constexpr int LDS = USED > (RG - 1) * kGradWaves * MERGE ? USED : (RG - 1) * kGradWaves * MERGE;
    __shared__ __attribute__((aligned(1024))) char smem[LDS];
    const int lane = threadIdx.x & 63, l31 = lane & 31, g = lane >> 5, blk = lane >> 4, s16 = lane & 15;
    const int wave_wg = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rgrp = RG == 1 ? 0 : wave_wg / kGradWaves, wave = wave_wg - rgrp * kGradWaves;
    char* const ring = smem + rgrp * 2 * STAGE;
    const int bh = (int)fastdiv(blockIdx.x, p.div_tiles_magic, p.div_tiles_shift);
    const int key0 = ((int)blockIdx.x - bh * p.tiles) * kGradTile;
    const int b = (int)fastdiv((unsigned)bh, p.div_h_magic, p.div_h_shift), h = bh - b * p.heads;
    int n = p.N;
    if (p.lens) {
        n = p.lens[b];
        n = n < 0 ? 0 : (n > p.N ? p.N : n);
    }
    const int key = key0 + wave * 32 + l31;
    const bool live = key < n;
    // this slice's chunks of rows, of all query heads one after the other; none where the tile has no key
    const int head_chunks = (p.M + RB - 1) / RB;
    const int all = key0 < n ? head_chunks * p.G : 0;
    const int per = (all + p.slices - 1) / p.slices;
    const int c0 = (int)blockIdx.y * per;
    const int chunks = all - c0 < per ? all - c0 : per;
    const int mine = (chunks - rgrp + RG - 1) / RG;      // chunk i of this group is c0 + i * RG + rgrp
    const int loops = (chunks + RG - 1) / RG;            // all groups take part in the barriers of the first

    const int q_rs = (int)p.q_rs, go_rs = (int)p.g_rs;
    const unsigned q_off = T::lane_offset(wave, lane, q_rs), go_off = T::lane_offset(wave, lane, go_rs);
    int head_at = 0, chunk_at = c0 + rgrp;               // of the next copy
    auto settle = [&]() __attribute__((always_inline)) {
        while (chunk_at >= head_chunks) {
            chunk_at -= head_chunks;
            ++head_at;
        }
    };
    if (chunks > 0) {
        head_at = chunk_at / head_chunks;
        chunk_at -= head_at * head_chunks;
    }
    auto copy = [&](int st_at) __attribute__((always_inline)) {
        char* const st = ring + st_at * STAGE;
        const int hq = h * p.G + head_at, m = chunk_at * RB, left = p.M - m;
        T::copy(st, (const char*)p.Q + 2 * (b * p.q_bs + (long long)m * q_rs + hq * p.q_hs), left, q_rs, q_off, wave, lane);
        T::copy(st + T::BYTES, (const char*)p.dO + 2 * (b * p.g_bs + (long long)m * go_rs + hq * p.g_hs), left, go_rs, go_off, wave, lane);
        const long long stat = ((long long)b * p.heads * p.G + hq) * p.M + m;
        // (the lanes past RB floats would write past their place)
        if (wave < 2 && lane < RB) floats_to_lds(make_rsrc32((wave ? p.delta : p.lse) + stat, (unsigned)(left < RB ? left : RB) * 4u), st + 2 * T::BYTES + wave * (RB * 4), (unsigned)lane * 4);
        chunk_at += RG;
        settle();
    };
    if (mine > 0) copy(0);
    if (V_LDS && rgrp == 0 && chunks > 0)
        VT::copy(smem + V_AT, (const char*)p.V + 2 * (b * p.v_bs + key0 * p.v_rs + h * p.v_hs), n - key0, (int)p.v_rs, VT::lane_offset(wave, lane, (int)p.v_rs), wave, lane);

    uint4 kf[KSTEPS], vf[V_LDS ? 1 : KSTEPS];
#pragma unroll
    for (int ks = 0; ks < KSTEPS; ++ks) kf[ks] = make_uint4(0, 0, 0, 0);
    if constexpr (!V_LDS)
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) vf[ks] = make_uint4(0, 0, 0, 0);
    if (live) {
        const char* const k = (const char*)p.K + 2 * (b * p.k_bs + key * p.k_rs + h * p.k_hs) + g * 16;
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) kf[ks] = *(const uint4*)(k + ks * 32);
        if constexpr (!V_LDS) {
            const char* const v = (const char*)p.V + 2 * (b * p.v_bs + key * p.v_rs + h * p.v_hs) + g * 16;
#pragma unroll
            for (int ks = 0; ks < KSTEPS; ++ks) vf[ks] = *(const uint4*)(v + ks * 32);
        }
    }
    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) dk[db][r] = dv[db][r] = 0.f;
    float by = DT == DT_F16 ? kFirstFactor : 1.f;
    const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    typedef float f32x4 __attribute__((ext_vector_type(4)));

    // (w holds the first part)
    unsigned w[8];
    auto second_part = [&](const char* tile, int ib, const f32x16& x, float factor, f32x16 (&to)[DB]) __attribute__((always_inline)) {
        if constexpr (TWO) {
            rest_of<DT>(x, factor, w);
            products<2 * DB, LA>([&](int t) __attribute__((always_inline)) { return T::across(tile, ib * 32 + t / DB * 16, t % DB, blk, s16); },
                                 [&](int t, const uint4& y) __attribute__((always_inline)) {
                                     const int ss = t / DB;
                                     to[t % DB] = InTraits<DT>::mfma(y, make_uint4(w[4 * ss], w[4 * ss + 1], w[4 * ss + 2], w[4 * ss + 3]), to[t % DB]);
                                 });
#pragma unroll
            for (int db = 0; db < DB; ++db) here(to[db]);
        }
    };

    for (int i = 0; i < loops; ++i) {
        copy_barrier<0>();
        if (i + 1 < mine) copy((i + 1) & 1);
        if (i >= mine) continue;               // (the longer group's last chunk)
        const char* const tq = ring + (i & 1) * STAGE;
        const char* const to = tq + T::BYTES;
#pragma unroll
        for (int ib = 0; ib < RB / 32; ++ib) {
            f32x16 pr;
            products<KSTEPS, LA>([&](int ks) __attribute__((always_inline)) { return T::along(tq, ib * 32, ks, l31, g); },
                                 [&](int ks, const uint4& x) __attribute__((always_inline)) { pr = InTraits<DT>::mfma(x, kf[ks], ks == 0 ? zero16 : pr); });
            // row 8*a + 4*g + e of the block is register 4*a + e.  Rows behind the last read zeros: P = 1 there, dO and dS are 0.
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                const f32x4 l4 = *(const f32x4*)(to + T::BYTES + (ib * 32 + 8 * a + 4 * g) * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    pr[4 * a + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(pr[4 * a + e], p.scale_log2e, __builtin_fmaf(l4[e], -1.44269504088896340736f, p_factor_log2<DT>())));
                w[2 * a] = grad_pack<DT>(pr[4 * a], pr[4 * a + 1]);
                w[2 * a + 1] = grad_pack<DT>(pr[4 * a + 2], pr[4 * a + 3]);
            }
            // dV of channel block t % DB from rows 16 * (t / DB) ..
            products<2 * DB, LA>([&](int t) __attribute__((always_inline)) { return T::across(to, ib * 32 + t / DB * 16, t % DB, blk, s16); },
                                 [&](int t, const uint4& x) __attribute__((always_inline)) {
                                     const int ss = t / DB;
                                     dv[t % DB] = InTraits<DT>::mfma(x, make_uint4(w[4 * ss], w[4 * ss + 1], w[4 * ss + 2], w[4 * ss + 3]), dv[t % DB]);
                                 });
#pragma unroll
            for (int db = 0; db < DB; ++db) here(dv[db]);
            second_part(to, ib, pr, 1.f, dv);
            f32x16 ds;
            if constexpr (V_LDS)
                products<KSTEPS, LA>([&](int ks) __attribute__((always_inline)) { return TwoOperands{T::along(to, ib * 32, ks, l31, g), VT::along(smem + V_AT, wave * 32, ks, l31, g)}; },
                                     [&](int ks, const TwoOperands& x) __attribute__((always_inline)) { ds = InTraits<DT>::mfma(x.a, x.b, ks == 0 ? zero16 : ds); });
            else
                products<KSTEPS, LA>([&](int ks) __attribute__((always_inline)) { return T::along(to, ib * 32, ks, l31, g); },
                                     [&](int ks, const uint4& x) __attribute__((always_inline)) { ds = InTraits<DT>::mfma(x, vf[ks], ks == 0 ? zero16 : ds); });
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                const f32x4 d4 = *(const f32x4*)(to + T::BYTES + RB * 4 + (ib * 32 + 8 * a + 4 * g) * 4);
#pragma unroll
                for (int e = 0; e < 4; ++e) ds[4 * a + e] = pr[4 * a + e] * (ds[4 * a + e] - d4[e]);
            }
            round_ds<DT, DB>(ds, by, dk, w);
            products<2 * DB, LA>([&](int t) __attribute__((always_inline)) { return T::across(tq, ib * 32 + t / DB * 16, t % DB, blk, s16); },
                                 [&](int t, const uint4& x) __attribute__((always_inline)) {
                                     const int ss = t / DB;
                                     dk[t % DB] = InTraits<DT>::mfma(x, make_uint4(w[4 * ss], w[4 * ss + 1], w[4 * ss + 2], w[4 * ss + 3]), dk[t % DB]);
                                 });
#pragma unroll
            for (int db = 0; db < DB; ++db) here(dk[db]);
            second_part(tq, ib, ds, by, dk);
        }
    }
    const float pf = DT == DT_F16 ? 0x1p-14f : 1.f;
    const float fk = n == 1 ? 0.f : p.scale * pf / by, fv = pf;      // (dS was formed from probabilities times their factor; that of a single key is zero)
    if constexpr (RG > 1) {
        __syncthreads();                                 // the rings are free
        f32x4* const o = (f32x4*)(smem + wave * MERGE) + lane;
        if (rgrp == 1) {
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    o[(db * 4 + q4) * 64] = f32x4{dk[db][4 * q4] * fk, dk[db][4 * q4 + 1] * fk, dk[db][4 * q4 + 2] * fk, dk[db][4 * q4 + 3] * fk};
                    o[((DB + db) * 4 + q4) * 64] = f32x4{dv[db][4 * q4] * fv, dv[db][4 * q4 + 1] * fv, dv[db][4 * q4 + 2] * fv, dv[db][4 * q4 + 3] * fv};
                }
        }
        __syncthreads();
        if (rgrp == 1) return;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const f32x4 x = o[(db * 4 + q4) * 64], y = o[((DB + db) * 4 + q4) * 64];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    dk[db][4 * q4 + e] = __builtin_fmaf(dk[db][4 * q4 + e], fk, x[e]);
                    dv[db][4 * q4 + e] = __builtin_fmaf(dv[db][4 * q4 + e], fv, y[e]);
                }
            }
    } else {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                dk[db][r] *= fk;
                dv[db][r] *= fv;
            }
    }
    char* const stage = smem + wave * (RG == 1 ? 32 * DH * 2 : MERGE);      // this wave's place for the 32 rows that it stores: where it read the other group's sums, or the first rings
    static_assert(RG > 1 || kGradWaves * 32 * DH * 2 <= LDS, "");
    if (p.slices > 1) {
        if (key0 + wave * 32 >= p.N) return;             // (nobody reads these)
        f32x4* const o = (f32x4*)(p.ws + ((long long)blockIdx.x * p.slices + blockIdx.y) * grad_partial(true, DH)) + wave * (32 * DH / 4) + lane;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                o[(db * 4 + q4) * 64] = f32x4{dk[db][4 * q4], dk[db][4 * q4 + 1], dk[db][4 * q4 + 2], dk[db][4 * q4 + 3]};
                o[(db * 4 + q4) * 64 + kGradTile * DH / 4] = f32x4{dv[db][4 * q4], dv[db][4 * q4 + 1], dv[db][4 * q4 + 2], dv[db][4 * q4 + 3]};
            }
        return;
    }
    // keys behind the sequence's have zeros
    auto store = [&](const f32x16 (&x)[DB], void* to, long long bs, long long rs, long long hs) __attribute__((always_inline)) {
        if constexpr (RG == 1) __syncthreads();          // the rings are free (the merged groups' values that were read last are each wave's own)
        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                const uint2 v = make_uint2(grad_pack<DT>(x[db][4 * q4], x[db][4 * q4 + 1]), grad_pack<DT>(x[db][4 * q4 + 2], x[db][4 * q4 + 3]));
                grad_stage<DH>(stage, l31, db * 32 + q4 * 8 + 4 * g, live ? v : make_uint2(0, 0));
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        const int first = key0 + wave * 32;
        grad_store<DH, 64>(stage, (unsigned short*)to + b * bs + first * rs + h * hs, p.N - first, true, [&](int r) __attribute__((always_inline)) -> long long { return r * rs; });
    };
    store(dk, p.dK, p.k_bs, p.k_rs, p.k_hs);
    store(dv, p.dV, p.v_bs, p.v_rs, p.v_hs);
}

// ---------------------------------------------------------------------------------------------
// The slices' partial sums, added in slice order: one thread per four values of a tile.  KEYS: dK (the first half of a partial) and dV.  Rows: dQ = sum of dS' K - e * sum of P K, and D.
// ---------------------------------------------------------------------------------------------
template <int DT, int DH, bool KEYS> __global__ void __launch_bounds__(256) grad_sum_kernel(const GradParams p) {
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    constexpr int PART = grad_partial(KEYS, DH) / 4, HALF = kGradTile * DH / 4;
    const int tile = (int)blockIdx.y, at = (int)(blockIdx.x * 256 + threadIdx.x);      // < (KEYS ? 2 : 1) * HALF: a multiple of 256
    const int bh = (int)fastdiv((unsigned)tile, p.div_tiles_magic, p.div_tiles_shift);
    const int b = (int)fastdiv((unsigned)bh, p.div_h_magic, p.div_h_shift), h = bh - b * p.heads;
    const int in = at % HALF, lane = in & 63, grp = in >> 6;       // grp = wave * (DH / 8) + db * 4 + quarter
    const int in_tile = grp / (DH / 8) * 32 + (lane & 31), row = (tile - bh * p.tiles) * kGradTile + in_tile;
    const int ch = grp % (DH / 8) * 8 + 4 * (lane >> 5);
    if (row >= (KEYS ? p.N : p.M * p.G)) return;                                    // (what no pass writes)
    const f32x4* const part = (const f32x4*)p.ws + (long long)tile * p.slices * PART + at;
    f32x4 sum = part[0];
    if constexpr (KEYS) {
#pragma unroll 4
        for (int z = 1; z < p.slices; ++z) sum += part[(long long)z * PART];
    } else {
        f32x4 pk = part[HALF];
        const float* const e_at = p.ws + (long long)tile * p.slices * (4 * PART) + 2 * kGradTile * DH + in_tile;
        float e = e_at[0];
#pragma unroll 4
        for (int z = 1; z < p.slices; ++z) {
            sum += part[(long long)z * PART];
            pk += part[(long long)z * PART + HALF];
            e += e_at[(long long)z * (4 * PART)];
        }
        sum -= e * pk;
        const int m = (int)fastdiv((unsigned)row, p.div_g_magic, p.div_g_shift), hq = h * p.G + row - m * p.G;
        if (ch == 0) p.delta[((long long)b * p.heads * p.G + hq) * p.M + m] += e;
        *(uint2*)((unsigned short*)p.dQ + b * p.q_bs + m * p.q_rs + hq * p.q_hs + ch) = make_uint2(grad_pack<DT>(sum[0], sum[1]), grad_pack<DT>(sum[2], sum[3]));
        return;
    }
    const uint2 v = make_uint2(grad_pack<DT>(sum[0], sum[1]), grad_pack<DT>(sum[2], sum[3]));
    int n = p.N;
    if (p.lens) {
        n = p.lens[b];
        n = n < 0 ? 0 : (n > p.N ? p.N : n);
    }
    unsigned short* const o = at >= HALF ? (unsigned short*)p.dV + b * p.v_bs + row * p.v_rs + h * p.v_hs : (unsigned short*)p.dK + b * p.k_bs + row * p.k_rs + h * p.k_hs;
    *(uint2*)(o + ch) = row < n ? v : make_uint2(0, 0);
}

}  // namespace tir
