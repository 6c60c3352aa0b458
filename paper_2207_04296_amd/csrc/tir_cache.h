// A paged cache of keys and values in 8 bits, and attention over it.
//
// Pools of blocks of T tokens (T = 16, 32, 64 or 128), one [T][d] tile of keys and one [d][T] tile of values per block and head, each with
// a scale of its own; a table gives every sequence its blocks.  The values' tiles are transposed because the second product of an
// attention, O^T = V^T P^T, contracts over the tokens: a lane's operand is 16 tokens of one channel, which is one 16-byte load this way.
#pragma once
#include "tir_kernel.h"

namespace tir {

enum : int { CT_I8 = 0, CT_E4M3 = 1 };

struct CacheView {
    char* k;                // [blocks][heads][T][d]
    char* v;                // [blocks][heads][d][T]
    float* ks;              // [blocks][heads]
    float* vs;
    const int* table;       // [batch][cols]
    int blocks, heads, cols, shift;      // T = 1 << shift
};

struct AppendParams {
    CacheView c;
    const void* K;          // new tokens: element (sequence, token, head, channel) at b*bs + t*rs + h*hs + channel
    const void* V;
    long long k_bs, k_rs, k_hs, v_bs, v_rs, v_hs;
    const int* start;       // tokens a sequence holds already
    const int* count;       // new tokens of a sequence, at most T; null: T each
    int T, touched;         // touched: blocks that T tokens can reach into
    unsigned div_h_magic, div_t_magic;      // / heads, / touched
    int div_h_shift, div_t_shift;
};

struct CacheAttnParams {
    CacheView c;
    const void* Q;
    void* O;
    long long q_bs, q_rs, q_hs, o_bs, o_rs, o_hs;
    const int* lens;        // tokens a sequence holds, the new ones among them
    const int* count;       // its queries, at most T; null: T each
    int T, G;               // query heads per key head
    int batch, tiles;       // tiles of queries per sequence and key head
    int rows_of_tile;       // which kernel: 16, 32, or 32 * kCacheTileWaves
    int slices;             // workgroups that share a tile's keys
    int out32;              // fp32 output
    float scale_log2e;
    void* ws;               // partial results: [tile][slice][kPartial] (slices > 1)
    unsigned* ws_count;     // [tile], zero between launches
    unsigned div_g_magic, div_h_magic, div_tiles_magic;      // / G, / heads, / tiles
    int div_g_shift, div_h_shift, div_tiles_shift;
};

constexpr int kCacheTileWaves = 8;

hipError_t launch_append(const AppendParams& p, int dt, int ct, int d, int64_t batch, hipStream_t stream);
hipError_t launch_cache_attention(const CacheAttnParams& p, int dt, int ct, int d, hipStream_t stream);

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------------------------
// Appending.
//
// Of a block and head that gets tokens: s = max(scale it has (0 if it holds no earlier token of the sequence), max|x| * (1/Q), 2^-64), Q the
// largest value of the 8-bit type; the new values are x * (1/s) rounded to that type, and where s grew the held ones are
// rounded again from q * (s_old * (1/s)).  Every operation is one binary32 operation, so that the result is one defined value.
// A value that is not finite counts as the nearest finite one, NaN as 0.
//
// One workgroup per sequence, block it reaches into, head, and keys or values: the scale needs all of the block's new values first.  They stay in
// registers between the two.  Bound by memory (2 bytes read and 1 written per value), for single tokens by latency.
// ---------------------------------------------------------------------------------------------
template <int CT> __device__ __forceinline__ float cache_step() { return CT == CT_I8 ? (float)(1.0 / 127.0) : (float)(1.0 / 448.0); }

// Four values, already times 1/s, as the bytes of a word.
template <int CT> __device__ __forceinline__ unsigned to_eight(float a, float b, float c, float d) {
    constexpr float top = CT == CT_I8 ? 127.0f : 448.0f;
    if constexpr (CT == CT_I8) {
        auto one = [](float x) __attribute__((always_inline)) { return (unsigned)(int)__builtin_amdgcn_fmed3f(__builtin_rintf(x), -top, top) & 255u; };
        return one(a) | one(b) << 8 | one(c) << 16 | one(d) << 24;
    } else {
        auto one = [](float x) __attribute__((always_inline)) { return __builtin_amdgcn_fmed3f(x, -top, top); };
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(one(a), one(b), 0, false);
        return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(one(c), one(d), lo, true);
    }
}
// Bytes I of a word as a value.
template <int CT> __device__ __forceinline__ void from_eight(unsigned w, float (&f)[4]) {
    if constexpr (CT == CT_I8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = (float)(signed char)(w >> (8 * i));
    } else {
        typedef float f2 __attribute__((ext_vector_type(2)));
        const f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        f[0] = lo[0]; f[1] = lo[1]; f[2] = hi[0]; f[3] = hi[1];
    }
}
template <int CT> __device__ __forceinline__ unsigned requantise(unsigned w, float ratio) {
    float f[4];
    from_eight<CT>(w, f);
    return to_eight<CT>(f[0] * ratio, f[1] * ratio, f[2] * ratio, f[3] * ratio);
}
// Eight 16-bit values as finite floats.
typedef float f32x8 __attribute__((ext_vector_type(8)));
template <int DT> __device__ __forceinline__ f32x8 finite8(const uint4& w) {
    f32x8 f;
    auto put = [&](int i, unsigned h) __attribute__((always_inline)) {
        float x;
        if constexpr (DT == DT_F16) x = (float)__builtin_bit_cast(_Float16, (unsigned short)h);
        else x = __builtin_bit_cast(float, h << 16);
        x = x == x ? x : 0.f;
        f[i] = __builtin_amdgcn_fmed3f(x, -__FLT_MAX__, __FLT_MAX__);
    };
    put(0, w.x & 0xffffu); put(1, w.x >> 16); put(2, w.y & 0xffffu); put(3, w.y >> 16);
    put(4, w.z & 0xffffu); put(5, w.z >> 16); put(6, w.w & 0xffffu); put(7, w.w >> 16);
    return f;
}

constexpr int kAppendThreads = 256;

template <int DT, int CT, int DH, int BT, bool KEYS> __device__ __forceinline__ void append_side(const AppendParams& p) {
    const int bj = (int)fastdiv(blockIdx.x, p.div_h_magic, p.div_h_shift);
    const int h = (int)blockIdx.x - bj * p.c.heads;
    const int b = (int)fastdiv((unsigned)bj, p.div_t_magic, p.div_t_shift);
    const int j = bj - b * p.touched;
    // positions first + lo .. first + hi - 1 of the sequence are this block's new tokens
    int start = p.start[b], cnt = p.count ? p.count[b] : p.T;
    start = start < 0 ? 0 : start;
    cnt = cnt < 0 ? 0 : (cnt > p.T ? p.T : cnt);
    const long long col = (long long)(start / BT) + j;
    if (col >= p.c.cols) return;
    const long long first = col * BT;
    const int lo = first > start ? 0 : (int)(start - first);                       // in the block
    const long long left = (long long)start + cnt - first;
    const int hi = left >= BT ? BT : (int)(left < 0 ? 0 : left);
    if (hi <= lo) return;
    const int id = p.c.table[(long long)b * p.c.cols + col];
    const long long rs = 2 * (KEYS ? p.k_rs : p.v_rs);
    // (token 0 of the block, which need not be a new one)
    const char* const src = (const char*)(KEYS ? p.K : p.V) + 2 * (b * (KEYS ? p.k_bs : p.v_bs) + h * (KEYS ? p.k_hs : p.v_hs)) + (first - start) * rs;

    // A thread's units.  Keys: 16 channels of one token, so that rows are read and written whole.  Values: 8 channels of 4 tokens, which are
    // one word of each of 8 of the tile's rows.  Either is two to four 16-byte loads, and 128 tokens of 128 channels are four or two units per thread.
    constexpr int UNITS = KEYS ? BT * DH / 16 : BT / 4 * DH / 8, U = (UNITS + kAppendThreads - 1) / kAppendThreads, L = KEYS ? 2 : 4;
    constexpr int KC = DH / 16, VG = BT / 4;
    uint4 w[U * L];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int q = (int)threadIdx.x + u * kAppendThreads;
#pragma unroll
        for (int e = 0; e < L; ++e) {
            const int tok = KEYS ? q / KC : q % VG * 4 + e;
            const int at = KEYS ? q % KC * 32 + e * 16 : q / VG * 16;
            w[u * L + e] = q < UNITS && tok >= lo && tok < hi ? *(const uint4*)(src + tok * rs + at) : make_uint4(0, 0, 0, 0);
        }
    }
    // (requested before the block's id is looked at: for a single token each trip to memory that waits for another is a fifth of the call)
    TIR_FENCE();
    if (id < 0 || id >= p.c.blocks) return;
    const long long bh = (long long)id * p.c.heads + h;
    float* const scale = (KEYS ? p.c.ks : p.c.vs) + bh;
    char* const tile = (KEYS ? p.c.k : p.c.v) + bh * (DH * BT);
    float was = 0.f;
    if (lo > 0) was = *scale;
    // words of values that are only partly new
    u32x4 part[KEYS ? 1 : 2 * U];
    if constexpr (!KEYS) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int q = (int)threadIdx.x + u * kAppendThreads, t0 = q % VG * 4;
            part[2 * u] = part[2 * u + 1] = u32x4{0, 0, 0, 0};
            if (q < UNITS && t0 < hi && t0 + 4 > lo && (t0 < lo || t0 + 4 > hi)) {
                const char* const at = tile + (q / VG * 8) * BT + t0;
#pragma unroll
                for (int i = 0; i < 8; ++i) part[2 * u + i / 4][i % 4] = *(const unsigned*)(at + i * BT);
            }
        }
    }
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < U * L; ++i) {
        const f32x8 f = finite8<DT>(w[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = __builtin_fmaxf(top, __builtin_fabsf(f[e]));
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, s));
    __shared__ float tops[kAppendThreads / 64];
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    const bool held = lo > 0;
    asm volatile("" : "+v"(was));                        // (the old scale is here before anybody writes the new one)
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kAppendThreads / 64; ++i) top = __builtin_fmaxf(top, tops[i]);
    float now = top * cache_step<CT>();
    now = __builtin_fmaxf(now, 0x1p-64f);
    now = __builtin_fmaxf(now, was);
    const float inv = 1.0f / now;
    const float ratio = was * inv;
    const bool grew = now > was && held;
    if (threadIdx.x == 0 && !(now == was && held)) *scale = now;

#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int q = (int)threadIdx.x + u * kAppendThreads;
        if constexpr (KEYS) {
            const int tok = q / KC, c = q % KC;
            uint4* const dst = (uint4*)(tile + tok * DH + c * 16);
            if (q < UNITS && tok >= lo && tok < hi) {
                const f32x8 f = finite8<DT>(w[2 * u]), e = finite8<DT>(w[2 * u + 1]);
                *dst = make_uint4(to_eight<CT>(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv), to_eight<CT>(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv),
                                  to_eight<CT>(e[0] * inv, e[1] * inv, e[2] * inv, e[3] * inv), to_eight<CT>(e[4] * inv, e[5] * inv, e[6] * inv, e[7] * inv));
            } else if (grew && tok < lo) {
                const uint4 t = *dst;
                *dst = make_uint4(requantise<CT>(t.x, ratio), requantise<CT>(t.y, ratio), requantise<CT>(t.z, ratio), requantise<CT>(t.w, ratio));
            }
        } else {
            const int t0 = q % VG * 4;
            char* const dst = tile + (q / VG * 8) * BT + t0;
            if (q < UNITS && t0 < hi && t0 + 4 > lo) {
                // bytes of the word that are new, and that are held and have to be rounded again
                unsigned fresh = 0, again = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (t0 + e >= lo && t0 + e < hi) fresh |= 255u << (8 * e);
                    if (t0 + e < lo && grew) again |= 255u << (8 * e);
                }
                const f32x8 f0 = finite8<DT>(w[4 * u]), f1 = finite8<DT>(w[4 * u + 1]), f2 = finite8<DT>(w[4 * u + 2]), f3 = finite8<DT>(w[4 * u + 3]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const unsigned o = to_eight<CT>(f0[i] * inv, f1[i] * inv, f2[i] * inv, f3[i] * inv);
                    const unsigned old = part[2 * u + i / 4][i % 4];
                    unsigned kept = old;
                    if (again) kept = (old & ~again) | (requantise<CT>(old, ratio) & again);
                    *(unsigned*)(dst + i * BT) = (kept & ~fresh) | (o & fresh);
                }
            } else if (grew && q < UNITS && t0 + 4 <= lo) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    unsigned* const at = (unsigned*)(dst + i * BT);
                    *at = requantise<CT>(*at, ratio);
                }
            }
        }
    }
}

template <int DT, int CT, int DH, int BT> __global__ void __launch_bounds__(kAppendThreads) cache_append_kernel(const AppendParams p) {
    if (blockIdx.y == 0) append_side<DT, CT, DH, BT, true>(p);
    else append_side<DT, CT, DH, BT, false>(p);
}

// ---------------------------------------------------------------------------------------------
// Attention over the cache.
//
// S^T = K Q^T and O^T = V^T P^T on 32x32x16 MFMAs as in the dense attention, one lane per query.  A key head's query heads and a
// sequence's new tokens share the tile of 32 rows: row t*G + g is token t of query head h*G + g.  Row i of the first operand may be any key, and the one
// taken is 16*((i>>2)&1) + 4*(i>>3) + (i&3): the lane of half-wave g then holds the scores of the 16 consecutive keys from 16*g, which are
// the tokens of one scale, and of one 16-byte load of a row of the values' tile.
//
// 8-bit values are exact in 16 bits, so the operands are converted as they are and the scales enter elsewhere: the keys' in the score (t = q.k * scale *
// ks, one factor per lane and chunk), the values' in the weight: w_j = p_j * vs_j is what is rounded for the second product, and the softmax runs on t_j + log2(vs_j), so that
// the largest weight of a row is one number whatever the scales are (p_j * vs_j with a p of at most 1 would leave binary16's normal range): 1, or 2^14 in binary16, which
// then holds weights down to 2^-28 of the largest to eleven bits; relative to 1 they would end at 2^-14, and a hundred thousand small weights rounded alike are seen in the sum.  The sum of probabilities takes each weight over its
// scale again: l = sum w_j / vs_j, in fp32.
// ---------------------------------------------------------------------------------------------
template <int DT, int CT> __device__ __forceinline__ uint2 widen(unsigned w) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    if constexpr (CT == CT_E4M3 && DT == DT_F16) {
        return make_uint2(__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false)),
                          __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true)));
    } else if constexpr (CT == CT_E4M3) {
        return make_uint2(__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)),
                          __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)));
    } else if constexpr (DT == DT_F16) {
        // x + 128 as the low bits of 1024 + x + 128 in binary16, less 1152
        const unsigned x = w ^ 0x80808080u;
        const h2 off = {(_Float16)1152.f, (_Float16)1152.f};
        return make_uint2(__builtin_bit_cast(unsigned, __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, x, 0x07010700u)) - off),
                          __builtin_bit_cast(unsigned, __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, x, 0x07030702u)) - off));
    } else {
        float f[4];
        from_eight<CT>(w, f);
        const b2 lo = {(__bf16)f[0], (__bf16)f[1]}, hi = {(__bf16)f[2], (__bf16)f[3]};
        return make_uint2(__builtin_bit_cast(unsigned, lo), __builtin_bit_cast(unsigned, hi));
    }
}
// Two of a 16-byte load's four words as the operand of one MFMA.
template <int DT, int CT> __device__ __forceinline__ uint4 widen8(unsigned a, unsigned b) {
    const uint2 lo = widen<DT, CT>(a), hi = widen<DT, CT>(b);
    return make_uint4(lo.x, lo.y, hi.x, hi.y);
}
// ... between the surrounding fences: the conversions of a chunk are not all done ahead, where their results would fill the registers.
template <int DT, int CT> __device__ __forceinline__ uint4 widen_here(unsigned a, unsigned b) {
    asm volatile("" : "+v"(a), "+v"(b));
    return widen8<DT, CT>(a, b);
}
template <int DT> __device__ __forceinline__ unsigned pack2(float a, float b) {
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
__device__ __forceinline__ float half_max(float x) {      // over the two half-waves
    const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    const unsigned lo = both[0], hi = both[1];
    return __builtin_fmaxf(__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi));
}

// log2 of the largest weight of a row
template <int DT> __device__ __forceinline__ float weight_bits() { return DT == DT_F16 ? 14.f : 0.f; }

// Partial results of a slice: a tile's accumulators, then its lanes' sums and references.
template <int DH> constexpr int cache_partial_bytes() { return DH / 32 * 4096 + 512; }

constexpr int kCacheWaves = 4;

template <int DT, int CT, int DH>
__global__ void __launch_bounds__(kCacheWaves * 64, 2) cache_rows_kernel(const CacheAttnParams p) {
    constexpr int KG = kCacheWaves, DB = DH / 32, KL = DH / 32;      // 16-byte loads per lane of a 32-key chunk: KL of the keys, DB of the values
    constexpr int MERGE = cache_partial_bytes<DH>();
    __shared__ __attribute__((aligned(1024))) char smem[KG * MERGE];
    const int lane = threadIdx.x & 63, l31 = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = (int)blockIdx.x, slice = (int)blockIdx.y;
    const int bh = (int)fastdiv((unsigned)tile, p.div_tiles_magic, p.div_tiles_shift);
    const int rt = tile - bh * p.tiles;
    const int b = (int)fastdiv((unsigned)bh, p.div_h_magic, p.div_h_shift);
    const int h = bh - b * p.c.heads;
    const int bt = 1 << p.c.shift;

    const long long cap = (long long)p.c.cols << p.c.shift;          // < 2^31: the host checks
    int len = p.lens[b], cnt = p.count ? p.count[b] : p.T;
    len = len < 0 ? 0 : (len > (int)cap ? (int)cap : len);
    cnt = cnt < 0 ? 0 : (cnt > p.T ? p.T : cnt);
    const int row0 = rt * 32;
    const int rows = cnt * p.G - row0;
    if (rows <= 0) return;
    // keys the rows of this tile see: up to the query's own position
    const int t_lane = (int)fastdiv((unsigned)(row0 + l31), p.div_g_magic, p.div_g_shift);
    const int g_lane = row0 + l31 - t_lane * p.G;
    const bool live = l31 < rows;
    const long long lim64 = (long long)len - cnt + t_lane + 1;
    const int lim = live ? (int)(lim64 < 0 ? 0 : lim64) : 0;
    const int t_first = (int)fastdiv((unsigned)row0, p.div_g_magic, p.div_g_shift);
    const int r_last = rows < 32 ? rows - 1 : 31;
    const int t_last = (int)fastdiv((unsigned)(row0 + r_last), p.div_g_magic, p.div_g_shift);
    const long long kmax64 = (long long)len - cnt + t_last + 1, kmin64 = (long long)len - cnt + t_first + 1;
    const int kmax = (int)(kmax64 < 0 ? 0 : kmax64), kmin = (int)(kmin64 < 0 ? 0 : kmin64);
    const int nch = (kmax + 31) >> 5;
    // this slice's chunks: at least two per wave
    int per = (nch + p.slices - 1) / p.slices;
    per = (per + KG - 1) / KG * KG;
    per = per < 2 * KG ? 2 * KG : per;
    const int active = nch > per ? (nch + per - 1) / per : 1;
    if (slice >= active) return;
    const int c_end = (slice + 1) * per < nch ? (slice + 1) * per : nch;
    const int c_first = slice * per + wave;
    const int mine = c_end > c_first ? (c_end - c_first + KG - 1) / KG : 0;

    uint4 qf[DH / 16];
    {
        const char* const q = (const char*)p.Q + 2 * (b * p.q_bs + t_lane * p.q_rs + (long long)(h * p.G + g_lane) * p.q_hs);
#pragma unroll
        for (int ks = 0; ks < DH / 16; ++ks)          // step 2*jj + s takes channels (2*jj + g)*16 + 8*s ..: the order of the keys' 16-byte loads
            qf[ks] = live ? *(const uint4*)(q + (((ks & ~1) + g) * 16 + (ks & 1) * 8) * 2) : make_uint4(0, 0, 0, 0);
    }
    f32x16 acc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] = 0.f;
    float m_run = -__FLT_MAX__, l_run = 0.f;

    const int krow = 16 * ((l31 >> 2) & 1) + 4 * (l31 >> 3) + (l31 & 3);      // this lane's key of a chunk
    const int* const table = p.c.table + (long long)b * p.c.cols;
    // Block ids of this wave's next 32 chunks, one granule of 16 tokens per lane
    auto fetch_ids = [&](int i0) __attribute__((always_inline)) -> int {
        const long long gran = 2ll * (c_first + (i0 + (lane >> 1)) * KG) + (lane & 1);
        const long long at = gran << 4 >> p.c.shift;
        return i0 + (lane >> 1) < mine && (gran << 4) < len ? table[at < p.c.cols ? at : p.c.cols - 1] : -1;
    };
    int ids = fetch_ids(0), ids_next = 0;

    struct Chunk {
        u32x4 k[KL], v[DB];
        float ks, vs;
        int bad;                    // this half-wave's granule has no block
    };
    auto load = [&](int i, Chunk& c) __attribute__((always_inline)) {
        const int at = (i & 31) * 2;
        const int id0 = __builtin_amdgcn_readlane(ids, at), id1 = __builtin_amdgcn_readlane(ids, at + 1);
        const bool ok0 = id0 >= 0 && id0 < p.c.blocks, ok1 = id1 >= 0 && id1 < p.c.blocks;
        const long long bh0 = (long long)(ok0 ? id0 : 0) * p.c.heads + h, bh1 = (long long)(ok1 ? id1 : 0) * p.c.heads + h;
        const int tok0 = (c_first + i * KG) * 32 & (bt - 1), tok1 = ((c_first + i * KG) * 32 + 16) & (bt - 1);      // in their blocks
        const long long k0 = ((bh0 << p.c.shift) + tok0) * DH, k1 = ((bh1 << p.c.shift) + tok1) * DH - 16 * DH;
        const char* const kp = p.c.k + ((l31 & 4) ? k1 : k0) + krow * DH + g * 16;
#pragma unroll
        for (int jj = 0; jj < KL; ++jj) c.k[jj] = *(const u32x4*)(kp + jj * 32);
        const long long v0 = ((bh0 * DH) << p.c.shift) + tok0, v1 = ((bh1 * DH) << p.c.shift) + tok1;
        const char* const vp = p.c.v + (g ? v1 : v0) + (l31 << p.c.shift);
#pragma unroll
        for (int db = 0; db < DB; ++db) c.v[db] = *(const u32x4*)(vp + ((db * 32) << p.c.shift));
        c.ks = p.c.ks[g ? bh1 : bh0];
        c.vs = p.c.vs[g ? bh1 : bh0];
        c.bad = !(g ? ok1 : ok0);
    };
    auto step = [&](int i, Chunk& c) __attribute__((always_inline)) {
        const int base = (c_first + i * KG) * 32;
        f32x16 s;
#pragma unroll
        for (int ks = 0; ks < DH / 16; ++ks) {
            const u32x4 w = c.k[ks >> 1];
            const uint4 kf = (ks & 1) ? widen_here<DT, CT>(w[2], w[3]) : widen_here<DT, CT>(w[0], w[1]);
            const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            s = InTraits<DT>::mfma(kf, qf[ks], ks == 0 ? zero : s);
            TIR_FENCE();                      // the next operand is widened under this product, and not earlier: its registers are short
        }
        const float vs = __builtin_fmaxf(c.vs, 0x1p-100f);
        const float mul = p.scale_log2e * c.ks, lvs = __builtin_amdgcn_logf(vs);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = __builtin_fmaf(s[r], mul, lvs);
        const bool ragged = base + 32 > kmin || __builtin_amdgcn_ballot_w64(c.bad) != 0;
        if (ragged) {
            const int n = c.bad ? 0 : lim - base - 16 * g;      // keys of the lane's sixteen that its row sees
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = r < n ? s[r] : -__builtin_inff();
            // what lies behind the sequence is not a value: e4m3 bytes there may be NaN, and NaN times a weight of zero is NaN
            if constexpr (CT == CT_E4M3) {
                const int nv = c.bad ? 0 : len - base - 16 * g;
                u32x4 keep;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int left = nv - 4 * e;
                    keep[e] = left >= 4 ? ~0u : (left <= 0 ? 0u : (1u << (8 * left)) - 1u);
                }
#pragma unroll
                for (int db = 0; db < DB; ++db) c.v[db] = c.v[db] & keep;
            }
        }
        float mx = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = __builtin_fmaxf(mx, s[r]);
        mx = __builtin_fmaxf(half_max(mx), -__FLT_MAX__);
        if (__builtin_amdgcn_ballot_w64(mx > m_run) != 0) {
            const float m_new = __builtin_fmaxf(m_run, mx);
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[db][r] *= alpha;
        }
        const float ref = m_run - weight_bits<DT>();
        float sum[2] = {0.f, 0.f};
        unsigned pw[8];
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
            float w[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                w[e] = __builtin_amdgcn_exp2f(s[r + e] - ref);
                sum[e] += w[e];
            }
            pw[r / 2] = pack2<DT>(w[0], w[1]);
        }
        l_run += (sum[0] + sum[1]) * __builtin_amdgcn_rcpf(vs);
#pragma unroll
        for (int ss = 0; ss < 2; ++ss) {
            const uint4 pf = make_uint4(pw[4 * ss], pw[4 * ss + 1], pw[4 * ss + 2], pw[4 * ss + 3]);
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                acc[db] = InTraits<DT>::mfma(widen_here<DT, CT>(c.v[db][2 * ss], c.v[db][2 * ss + 1]), pf, acc[db]);
                TIR_FENCE();
            }
        }
    };
    // chunk i + 1 is on its way while chunk i is worked on; the ids of the next 32 chunks likewise
    Chunk even, odd;
    if (mine > 0) load(0, even);
    for (int i = 0; i < mine; i += 2) {
        if ((i & 31) == 0) ids_next = fetch_ids(i + 32);
        if (i + 1 < mine) load(i + 1, odd);
        step(i, even);
        if (((i + 2) & 31) == 0) ids = ids_next;
        if (i + 2 < mine) load(i + 2, even);
        if (i + 1 < mine) step(i + 1, odd);
    }

    // ------------------------------------------------------------ the waves' results, relative to the largest reference
    constexpr int NG = DB * 4 / KG;                      // groups of four channels this wave finishes
    static_assert(NG * KG == DB * 4, "");
    f32x4 out[NG];
    float top, l;
    auto join = [&]() __attribute__((always_inline)) {
        f32x4* const o = (f32x4*)(smem + wave * MERGE);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) {
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = acc[db][4 * q4 + e];
                o[(db * 4 + q4) * 64 + lane] = v;
            }
        float* const t = (float*)(smem + wave * MERGE + DB * 4096);
        t[lane] = l_run;
        t[64 + lane] = m_run;
        __syncthreads();
        float f[KG];
        top = -__FLT_MAX__;
        l = 0.f;
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            f[k] = ((const float*)(smem + k * MERGE + DB * 4096))[64 + lane];
            top = __builtin_fmaxf(top, f[k]);
        }
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            f[k] = __builtin_amdgcn_exp2f(f[k] - top);
            l += f[k] * ((const float*)(smem + k * MERGE + DB * 4096))[lane];
        }
#pragma unroll
        for (int n = 0; n < NG; ++n) {
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KG; ++k) v += f[k] * ((const f32x4*)(smem + k * MERGE))[(wave * NG + n) * 64 + lane];
            out[n] = v;
        }
    };
    l_run += __shfl_xor(l_run, 32);
    join();
    if (active > 1) {
        // Slices of a tile: as for the split reduction of a product, the partial results go through memory at system scope, the last to
        // arrive adds them in an order of their own: each wave its share of the slices (one after the other a load's trip to memory per slice would be seen), then the waves.
        constexpr int kSystemScope = 17;
        const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc((char*)p.ws + (long long)tile * p.slices * MERGE, 0, p.slices * MERGE, 0x00020000);
#pragma unroll
        for (int n = 0; n < NG; ++n)
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, out[n]), rw, ((wave * NG + n) * 64 + lane) * 16, slice * MERGE, kSystemScope);
        if (wave == 0) {
            __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, l), rw, DB * 4096 + lane * 4, slice * MERGE, kSystemScope);
            __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, top), rw, DB * 4096 + 256 + lane * 4, slice * MERGE, kSystemScope);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        unsigned* const flag = (unsigned*)smem;
        if (threadIdx.x == 0) *flag = __hip_atomic_fetch_add(p.ws_count + tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
        __syncthreads();
        const bool last = *flag == (unsigned)active - 1u;
        __syncthreads();                                 // (the flag's place is the first wave's again)
        if (!last) return;
        if (threadIdx.x == 0) __hip_atomic_store(p.ws_count + tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
        const int at_l = DB * 4096 + lane * 4;
        auto load_ref = [&](int z) __attribute__((always_inline)) -> float {      // of a slice behind the last one: no weight
            const float m = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rw, z < active ? at_l + 256 : (int)kOutOfRange, z * MERGE, kSystemScope));
            return z < active ? m : -__FLT_MAX__;
        };
        m_run = -__FLT_MAX__;
        constexpr int Z = 8;
        for (int z0 = wave; z0 < active; z0 += KG * Z) {
            float m[Z];
#pragma unroll
            for (int z = 0; z < Z; ++z) m[z] = load_ref(z0 + z * KG);
#pragma unroll
            for (int z = 0; z < Z; ++z) m_run = __builtin_fmaxf(m_run, m[z]);
        }
        l_run = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[db][r] = 0.f;
        constexpr int W = 2;                             // slices on their way at a time
        for (int z0 = wave; z0 < active; z0 += KG * W) {
            float m[W], ls[W];
            u32x4 v[W][DB * 4];
#pragma unroll
            for (int z = 0; z < W; ++z) {
                const int at = z0 + z * KG;
                m[z] = load_ref(at);
                ls[z] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rw, at < active ? at_l : (int)kOutOfRange, at * MERGE, kSystemScope));
#pragma unroll
                for (int n = 0; n < DB * 4; ++n)
                    v[z][n] = __builtin_amdgcn_raw_buffer_load_b128(rw, at < active ? (n * 64 + lane) * 16 : (int)kOutOfRange, at * MERGE, kSystemScope);
            }
#pragma unroll
            for (int z = 0; z < W; ++z) {
                const float f = z0 + z * KG < active ? __builtin_amdgcn_exp2f(m[z] - m_run) : 0.f;
                l_run += f * ls[z];
#pragma unroll
                for (int n = 0; n < DB * 4; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const unsigned t = v[z][n][e];
                        acc[n >> 2][(n & 3) * 4 + e] += f * __builtin_bit_cast(float, t);
                    }
            }
        }
        join();
    }
    if (!live) return;
    const float inv = lim > 0 && l != 0.f ? 1.0f / l : 0.f;           // a row that sees no key is zero
    const long long at = b * p.o_bs + t_lane * p.o_rs + (long long)(h * p.G + g_lane) * p.o_hs;
#pragma unroll
    for (int n = 0; n < NG; ++n) {
        const int grp = wave * NG + n, ch = grp / 4 * 32 + grp % 4 * 8 + 4 * g;
        const f32x4 v = out[n] * inv;
        if (p.out32) *(f32x4*)((float*)p.O + at + ch) = v;
        else *(uint2*)((unsigned short*)p.O + at + ch) = make_uint2(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]));
    }
}

// ---------------------------------------------------------------------------------------------
// The same for up to 16 rows of a key head, a token's query heads for instance, on 16x16x32 MFMAs: half the products and exponentials of the tile of 32, and chunks of 64 keys in the same registers.
//
// Lane l is query l & 15; its group q = l >> 4 holds the scores of the 16 keys from 16*q: tile j of four has row i as key 16*(i >> 2) + 4*j + (i & 3), and rows 4*q .. 4*q + 3 come out in
// group q.  A load instruction takes 64 consecutive bytes of 16 rows, of keys or of values, where the tile of 32 takes 32 bytes of 32: one token over 200 003, blocks of 128 tokens, 110 us there.
// ---------------------------------------------------------------------------------------------
template <int DT> __device__ __forceinline__ f32x4 mfma16(const uint4& a, const uint4& b, f32x4 c) {
    if constexpr (DT == DT_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// Partial results of a slice: accumulators [DH / 16][64] of four, sums and references [64].
template <int DH> constexpr int token_partial_bytes() { return DH / 16 * 1024 + 512; }

template <int DT, int CT, int DH>
__global__ void __launch_bounds__(kCacheWaves * 64, 2) cache_token_kernel(const CacheAttnParams p) {
    constexpr int KG = kCacheWaves, CB = DH / 16, KP = DH / 64;      // channel blocks of 16; 16-byte loads of a key per lane
    constexpr int MERGE = token_partial_bytes<DH>();
    __shared__ __attribute__((aligned(1024))) char smem[KG * MERGE];
    const int lane = threadIdx.x & 63, l15 = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = (int)blockIdx.x, slice = (int)blockIdx.y;       // one tile per sequence and key head
    const int b = (int)fastdiv((unsigned)tile, p.div_h_magic, p.div_h_shift);
    const int h = tile - b * p.c.heads;
    const int bt = 1 << p.c.shift;

    const long long cap = (long long)p.c.cols << p.c.shift;
    int len = p.lens[b], cnt = p.count ? p.count[b] : p.T;
    len = len < 0 ? 0 : (len > (int)cap ? (int)cap : len);
    cnt = cnt < 0 ? 0 : (cnt > p.T ? p.T : cnt);
    if (cnt == 0) return;
    const int t_lane = (int)fastdiv((unsigned)l15, p.div_g_magic, p.div_g_shift), g_lane = l15 - t_lane * p.G;
    const bool live = l15 < cnt * p.G;
    const int lim = live ? len - cnt + t_lane + 1 : 0;                // keys this lane's query sees, none if not above 0
    const int kmax = len, kmin = len - cnt + 1;                       // of the last query, and of the first (may be negative)
    const int nch = (kmax + 63) >> 6;
    int per = (nch + p.slices - 1) / p.slices;
    per = (per + KG - 1) / KG * KG;                                   // one chunk per wave at least
    const int active = nch > per ? (nch + per - 1) / per : 1;
    if (slice >= active) return;
    const int c_end = (slice + 1) * per < nch ? (slice + 1) * per : nch;
    const int c_first = slice * per + wave;
    const int mine = c_end > c_first ? (c_end - c_first + KG - 1) / KG : 0;

    const int* const table = p.c.table + (long long)b * p.c.cols;
    // Block ids of this wave's next 16 chunks, one granule of 16 tokens per lane
    auto fetch_ids = [&](int i0) __attribute__((always_inline)) -> int {
        const int i = i0 + (lane >> 2), tok = (c_first + i * KG) * 64 + (lane & 3) * 16;
        return i < mine && tok < len ? table[tok >> p.c.shift] : -1;
    };
    int ids = fetch_ids(0), ids_next = 0;

    uint4 qf[2 * KP];
    {
        const char* const q = (const char*)p.Q + 2 * (b * p.q_bs + t_lane * p.q_rs + (long long)(h * p.G + g_lane) * p.q_hs);
#pragma unroll
        for (int ks = 0; ks < 2 * KP; ++ks)           // step 2*k + s takes channels 64*k + 16*grp + 8*s ..: the order of the keys' 16-byte loads
            qf[ks] = live ? *(const uint4*)(q + ((ks >> 1) * 64 + grp * 16 + (ks & 1) * 8) * 2) : make_uint4(0, 0, 0, 0);
    }
    f32x4 acc[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) acc[cb] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -__FLT_MAX__, l_run = 0.f;

    const unsigned block_bytes = (unsigned)(p.c.heads * DH) << p.c.shift;
    const char* const pool_k = p.c.k + ((unsigned)(h * DH) << p.c.shift);
    const char* const pool_v = p.c.v + ((unsigned)(h * DH) << p.c.shift);
    struct Chunk {
        u32x4 k[4][KP], v[CB];
        float ks, vs;
        int bad;                    // this group's granule has no block
    };
    auto load = [&](int i, Chunk& c) __attribute__((always_inline)) {
        const int at = (i & 15) * 4, tok = (c_first + i * KG) * 64;
        const int idk = __shfl(ids, at + (l15 >> 2)), idv = __shfl(ids, at + grp);
        const bool okk = (unsigned)idk < (unsigned)p.c.blocks, okv = (unsigned)idv < (unsigned)p.c.blocks;
        const char* const kp = pool_k + (unsigned long long)(unsigned)(okk ? idk : 0) * block_bytes + (unsigned)(((tok + (l15 >> 2) * 16) & (bt - 1)) * DH + (l15 & 3) * DH + grp * 16);
        const char* const vp = pool_v + (unsigned long long)(unsigned)(okv ? idv : 0) * block_bytes + (unsigned)(((tok + grp * 16) & (bt - 1)) + (l15 << p.c.shift));
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int k = 0; k < KP; ++k) c.k[j][k] = *(const u32x4*)(kp + j * 4 * DH + k * 64);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            c.v[cb] = *(const u32x4*)(vp + ((cb * 16) << p.c.shift));
            TIR_FENCE();                      // (an address at a time)
        }
        const long long s = (long long)(okv ? idv : 0) * p.c.heads + h;
        c.ks = p.c.ks[s];
        c.vs = p.c.vs[s];
        c.bad = !okv;
    };
    auto over_groups = [](float x) __attribute__((always_inline)) -> float {
        const auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
        const unsigned lo = a[0], hi = a[1];
        return half_max(__builtin_fmaxf(__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi)));
    };
    auto step = [&](int i, Chunk& c) __attribute__((always_inline)) {
        const int base = (c_first + i * KG) * 64 + grp * 16;      // of this group's keys
        f32x4 s[4];
#pragma unroll
        for (int ks = 0; ks < 2 * KP; ++ks)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const u32x4 w = c.k[j][ks >> 1];
                const uint4 kf = (ks & 1) ? widen_here<DT, CT>(w[2], w[3]) : widen_here<DT, CT>(w[0], w[1]);
                s[j] = mfma16<DT>(kf, qf[ks], ks == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[j]);
                TIR_FENCE();
            }
        const float vs = __builtin_fmaxf(c.vs, 0x1p-100f);
        const float mul = p.scale_log2e * c.ks, lvs = __builtin_amdgcn_logf(vs);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[j][r] = __builtin_fmaf(s[j][r], mul, lvs);
        if (base - grp * 16 + 64 > kmin || __builtin_amdgcn_ballot_w64(c.bad) != 0) {
            const int n = c.bad ? 0 : lim - base;                 // keys of the lane's sixteen that its query sees (may be negative)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) s[j][r] = 4 * j + r < n ? s[j][r] : -__builtin_inff();
            if constexpr (CT == CT_E4M3) {                        // (as in the tile of 32: NaN bytes behind the sequence)
                const int nv = c.bad ? 0 : len - base;
                u32x4 keep;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int left = nv - 4 * e;
                    keep[e] = left >= 4 ? ~0u : (left <= 0 ? 0u : (1u << (8 * left)) - 1u);
                }
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) c.v[cb] = c.v[cb] & keep;
            }
        }
        float mx = s[0][0];
#pragma unroll
        for (int e = 1; e < 16; ++e) mx = __builtin_fmaxf(mx, s[e >> 2][e & 3]);
        mx = __builtin_fmaxf(over_groups(mx), -__FLT_MAX__);
        if (__builtin_amdgcn_ballot_w64(mx > m_run) != 0) {
            const float m_new = __builtin_fmaxf(m_run, mx);
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[cb][r] *= alpha;
        }
        const float ref = m_run - weight_bits<DT>();
        float sum[2] = {0.f, 0.f};
        unsigned pw[8];
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            float w[2];
#pragma unroll
            for (int z = 0; z < 2; ++z) {
                w[z] = __builtin_amdgcn_exp2f(s[e >> 2][(e & 3) + z] - ref);
                sum[z] += w[z];
            }
            pw[e / 2] = pack2<DT>(w[0], w[1]);
        }
        l_run += (sum[0] + sum[1]) * __builtin_amdgcn_rcpf(vs);
#pragma unroll
        for (int ss = 0; ss < 2; ++ss) {              // keys 16*grp + 8*ss ..
            const uint4 pf = make_uint4(pw[4 * ss], pw[4 * ss + 1], pw[4 * ss + 2], pw[4 * ss + 3]);
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                acc[cb] = mfma16<DT>(widen_here<DT, CT>(c.v[cb][2 * ss], c.v[cb][2 * ss + 1]), pf, acc[cb]);
                TIR_FENCE();
            }
        }
    };
    Chunk even, odd;
    // (behind the last chunk there is no block, and a load takes the pool's first: without a branch around the loads the two chunks need no copies)
    load(0, even);
    for (int i = 0; i < mine; i += 2) {
        if ((i & 15) == 0) ids_next = fetch_ids(i + 16);
        load(i + 1, odd);
        step(i, even);
        if (((i + 2) & 15) == 0) ids = ids_next;
        load(i + 2, even);
        if (i + 1 < mine) step(i + 1, odd);
    }

    // ------------------------------------------------------------ the waves' results, and the slices', as in the tile of 32
    constexpr int NG = CB / KG;                       // channel blocks this wave finishes
    static_assert(NG * KG == CB, "");
    f32x4 out[NG];
    float top, l;
    auto join = [&]() __attribute__((always_inline)) {
        f32x4* const o = (f32x4*)(smem + wave * MERGE);
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) o[cb * 64 + lane] = acc[cb];
        float* const t = (float*)(smem + wave * MERGE + CB * 1024);
        t[lane] = l_run;
        t[64 + lane] = m_run;
        __syncthreads();
        float f[KG];
        top = -__FLT_MAX__;
        l = 0.f;
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            f[k] = ((const float*)(smem + k * MERGE + CB * 1024))[64 + lane];
            top = __builtin_fmaxf(top, f[k]);
        }
#pragma unroll
        for (int k = 0; k < KG; ++k) {
            f[k] = __builtin_amdgcn_exp2f(f[k] - top);
            l += f[k] * ((const float*)(smem + k * MERGE + CB * 1024))[lane];
        }
#pragma unroll
        for (int n = 0; n < NG; ++n) {
            f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KG; ++k) v += f[k] * ((const f32x4*)(smem + k * MERGE))[(wave * NG + n) * 64 + lane];
            out[n] = v;
        }
    };
    l_run += __shfl_xor(l_run, 16);
    l_run += __shfl_xor(l_run, 32);
    join();
    if (active > 1) {
        constexpr int kSystemScope = 17;
        const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc((char*)p.ws + (long long)tile * p.slices * MERGE, 0, p.slices * MERGE, 0x00020000);
#pragma unroll
        for (int n = 0; n < NG; ++n)
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, out[n]), rw, ((wave * NG + n) * 64 + lane) * 16, slice * MERGE, kSystemScope);
        if (wave == 0) {
            __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, l), rw, CB * 1024 + lane * 4, slice * MERGE, kSystemScope);
            __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, top), rw, CB * 1024 + 256 + lane * 4, slice * MERGE, kSystemScope);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        unsigned* const flag = (unsigned*)smem;
        if (threadIdx.x == 0) *flag = __hip_atomic_fetch_add(p.ws_count + tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
        __syncthreads();
        const bool last = *flag == (unsigned)active - 1u;
        __syncthreads();
        if (!last) return;
        if (threadIdx.x == 0) __hip_atomic_store(p.ws_count + tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
        const int at_l = CB * 1024 + lane * 4;
        auto load_ref = [&](int z) __attribute__((always_inline)) -> float {
            const float m = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rw, z < active ? at_l + 256 : (int)kOutOfRange, z * MERGE, kSystemScope));
            return z < active ? m : -__FLT_MAX__;
        };
        m_run = -__FLT_MAX__;
        constexpr int Z = 8;
        for (int z0 = wave; z0 < active; z0 += KG * Z) {
            float m[Z];
#pragma unroll
            for (int z = 0; z < Z; ++z) m[z] = load_ref(z0 + z * KG);
#pragma unroll
            for (int z = 0; z < Z; ++z) m_run = __builtin_fmaxf(m_run, m[z]);
        }
        l_run = 0.f;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) acc[cb] = f32x4{0.f, 0.f, 0.f, 0.f};
        constexpr int W = 2;                          // slices on their way at a time
        for (int z0 = wave; z0 < active; z0 += KG * W) {
            float m[W], ls[W];
            u32x4 v[W][CB];
#pragma unroll
            for (int z = 0; z < W; ++z) {
                const int at = z0 + z * KG;
                m[z] = load_ref(at);
                ls[z] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rw, at < active ? at_l : (int)kOutOfRange, at * MERGE, kSystemScope));
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) v[z][cb] = __builtin_amdgcn_raw_buffer_load_b128(rw, at < active ? (cb * 64 + lane) * 16 : (int)kOutOfRange, at * MERGE, kSystemScope);
            }
#pragma unroll
            for (int z = 0; z < W; ++z) {
                const float f = z0 + z * KG < active ? __builtin_amdgcn_exp2f(m[z] - m_run) : 0.f;
                l_run += f * ls[z];
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) acc[cb] += f * __builtin_bit_cast(f32x4, v[z][cb]);
            }
        }
        join();
    }
    if (!live) return;
    const float inv = lim > 0 && l != 0.f ? 1.0f / l : 0.f;           // a row that sees no key is zero
    const long long at = b * p.o_bs + t_lane * p.o_rs + (long long)(h * p.G + g_lane) * p.o_hs;
#pragma unroll
    for (int n = 0; n < NG; ++n) {
        const int ch = (wave * NG + n) * 16 + 4 * grp;
        const f32x4 v = out[n] * inv;
        if (p.out32) *(f32x4*)((float*)p.O + at + ch) = v;
        else *(uint2*)((unsigned short*)p.O + at + ch) = make_uint2(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]));
    }
}

// ---------------------------------------------------------------------------------------------
// The same for many rows: QW waves of 32 rows each over chunks of 64 keys, which the workgroup widens to 16 bits once, on their way from registers into LDS, instead of every wave
// for itself (a wave that widens all it multiplies spends 160 instructions of a chunk's 400 on it).  K [64 keys][128 bytes] per 64 channels and V [channels][128 bytes of keys], both read along their
// rows; 16-byte column c of row r at column c ^ swizzle(r), which spreads the 16 rows of a read phase over all banks: rows 0-3, 16-19, 4-7, 20-23 of K (the order above), 0-15 of V.
//
// A wave runs its vector work under its own products, as in the dense attention: the exponentials of chunk i and the widening of what comes next stand between the MFMAs of K Q^T of chunk i + 1, the row
// maxima of that chunk between those of V^T P^T of chunk i.  Keys are therefore widened two chunks ahead of their weights and values one; what is widened was requested an iteration before, its block ids
// one more.
// ---------------------------------------------------------------------------------------------
// How a tile's chunks are shared among workgroups: runs of at least four.
struct TileShare {
    int chunks, per, active;
};
__device__ __forceinline__ TileShare tile_share(int kmax, int slices) {
    TileShare s;
    s.chunks = (kmax + 63) >> 6;
    s.per = (s.chunks + slices - 1) / slices;
    s.per = slices > 1 && s.per < 4 ? 4 : s.per;
    s.active = s.chunks > s.per ? (s.chunks + s.per - 1) / s.per : 1;
    return s;
}

template <int DT, int CT, int DH, int QW>
__global__ void __launch_bounds__(QW * 64, 2) cache_tile_kernel(const CacheAttnParams p) {
    constexpr int NT = QW * 64, TQ = QW * 32, DB = DH / 32, KSTEPS = DH / 16;
    constexpr int KBYTES = 64 * DH * 2, VBYTES = DH * 128;
    constexpr int HALF_UNITS = 64 * DH / 16, U = 2 * HALF_UNITS / NT;      // 16-byte units of the keys or values of a chunk; units per thread
    static_assert(U >= 1 && U * NT == 2 * HALF_UNITS, "");
    __shared__ __attribute__((aligned(1024))) char smem[2 * KBYTES + 2 * VBYTES + 4 * 64];
    char* const lds_v = smem + 2 * KBYTES;
    char* const lds_s = lds_v + 2 * VBYTES;                                // four chunks' scales: {factor of the scores, log2(vs), 1 / vs} of each granule of 16 tokens
    const int tid = (int)threadIdx.x, lane = tid & 63, l31 = lane & 31, g = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int bh = (int)fastdiv(blockIdx.x, p.div_tiles_magic, p.div_tiles_shift);
    const int row0 = ((int)blockIdx.x - bh * p.tiles) * TQ;
    const int b = (int)fastdiv((unsigned)bh, p.div_h_magic, p.div_h_shift);
    const int h = bh - b * p.c.heads;
    const int bt = 1 << p.c.shift;
    const long long cap = (long long)p.c.cols << p.c.shift;
    int len = p.lens[b], cnt = p.count ? p.count[b] : p.T;
    len = len < 0 ? 0 : (len > (int)cap ? (int)cap : len);
    cnt = cnt < 0 ? 0 : (cnt > p.T ? p.T : cnt);
    const int rows = cnt * p.G - row0;
    if (rows <= 0) return;
    auto seen_by = [&](int row) __attribute__((always_inline)) -> int {      // keys that a row of the sequence sees
        const long long n = (long long)len - cnt + (int)fastdiv((unsigned)row, p.div_g_magic, p.div_g_shift) + 1;
        return n < 0 ? 0 : (int)n;
    };
    const int kmax = seen_by(row0 + (rows < TQ ? rows : TQ) - 1);            // of the tile
    const TileShare share = tile_share(kmax, p.slices);
    if ((int)blockIdx.y >= share.active) return;
    const int c0 = (int)blockIdx.y * share.per;                              // this workgroup's chunks: c0 .. c1 - 1
    const int c1 = c0 + share.per < share.chunks ? c0 + share.per : share.chunks;
    const int row = row0 + wave * 32 + l31;
    const bool live = wave * 32 + l31 < rows;
    const int t_lane = (int)fastdiv((unsigned)row, p.div_g_magic, p.div_g_shift), g_lane = row - t_lane * p.G;
    const int lim = live ? seen_by(row) : kmax;                              // (rows behind the last one take part and are dropped)
    const int wmin = wave * 32 < rows ? seen_by(row0 + wave * 32) : kmax;    // from where on a chunk needs the wave's limits

    // ------------------------------------------------------------ from the pool to LDS
    // Unit u of this thread: 16 channels of a key (keys) or a channel's 16 keys (values).  Where a side has fewer units than threads, each half of the waves has one side.
    const int* const table = p.c.table + (long long)b * p.c.cols;
    auto is_key = [&](int u) __attribute__((always_inline)) -> bool { return HALF_UNITS >= NT ? u * NT < HALF_UNITS : wave < QW / 2; };
    auto unit = [&](int u) __attribute__((always_inline)) -> int { return (tid + u * NT) & (HALF_UNITS - 1); };
    auto granule = [&](int u) __attribute__((always_inline)) -> int { return is_key(u) ? unit(u) / KSTEPS >> 4 : unit(u) & 3; };
    auto block_of = [&](int i, int gr) __attribute__((always_inline)) -> int {      // block of granule gr of chunk i, or -1
        const int tok = i * 64 + gr * 16;            // (below 2^31: the table's columns end before)
        return tok < kmax ? table[tok >> p.c.shift] : -1;
    };
    const unsigned block_bytes = (unsigned)(p.c.heads * DH) << p.c.shift;      // of one block in either pool: at most 65535 * 128 * 128
    const char* const pool_k = p.c.k + ((unsigned)(h * DH) << p.c.shift);
    const char* const pool_v = p.c.v + ((unsigned)(h * DH) << p.c.shift);
    // the unit's place in a tile, less the tokens from the tile's start to the granule
    unsigned off[U];
#pragma unroll
    for (int u = 0; u < U; ++u) off[u] = is_key(u) ? (unsigned)(unit(u) / KSTEPS % 16 * DH + unit(u) % KSTEPS * 16) : (unsigned)(unit(u) >> 2) << p.c.shift;
    int ids[U], sid = -1, ok[U], sok = 0;
    u32x4 w[U];
    float ks = 0.f, vs = 0.f;
    // keys and scales of chunk ck, values of chunk cv
    auto fetch_ids = [&](int ck, int cv) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) ids[u] = block_of(is_key(u) ? ck : cv, granule(u));
        if (tid < 4) sid = block_of(ck, tid);
    };
    auto fetch = [&](int ck, int cv) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            ok[u] = (unsigned)ids[u] < (unsigned)p.c.blocks;
            const unsigned first = (unsigned)(((is_key(u) ? ck : cv) * 64 + granule(u) * 16) & (bt - 1));      // the granule's first token in its block
            const unsigned long long at = (unsigned long long)(unsigned)(ok[u] ? ids[u] : 0) * block_bytes + (off[u] + (is_key(u) ? first * DH : first));
            w[u] = *(const u32x4*)((is_key(u) ? pool_k : pool_v) + at);
        }
        if (tid < 4) {
            sok = (unsigned)sid < (unsigned)p.c.blocks;
            const long long base = (long long)(sok ? sid : 0) * p.c.heads + h;
            ks = p.c.ks[base];
            vs = p.c.vs[base];
        }
    };
    const float sc = __builtin_fabsf(p.scale_log2e);      // (a negative scale is a positive one on negated queries)
    auto swz_k = [](int r) __attribute__((always_inline)) { return ((r >> 1) & 3) | ((r >> 4) & 1) << 2; };
    auto put_unit = [&](int u, int ck, int cv) __attribute__((always_inline)) {
        const int q = unit(u);
        u32x4 x = w[u];
        if (is_key(u)) {
            const int key = q / KSTEPS, c = q % KSTEPS;      // channels 16*c ..
            // what lies behind the sequence is no value: zeros, whatever the bytes say
            if (!ok[u] || ck * 64 + key >= len) x = u32x4{0, 0, 0, 0};
            char* const at = smem + (ck & 1) * KBYTES + (c >> 2) * (64 * 128) + key * 128;
            *(uint4*)(at + ((((c & 3) * 2) ^ swz_k(key)) << 4)) = widen_here<DT, CT>(x[0], x[1]);
            *(uint4*)(at + ((((c & 3) * 2 + 1) ^ swz_k(key)) << 4)) = widen_here<DT, CT>(x[2], x[3]);
        } else {
            const int ch = q >> 2, gr = q & 3;
            const int nv = ok[u] ? len - cv * 64 - gr * 16 : 0;
            if (nv < 16) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int left = nv - 4 * e;
                    x[e] &= left >= 4 ? ~0u : (left <= 0 ? 0u : (1u << (8 * left)) - 1u);
                }
            }
            char* const at = lds_v + (cv & 1) * VBYTES + ch * 128;
            *(uint4*)(at + (((gr * 2) ^ kmajor_swz<128>(ch)) << 4)) = widen_here<DT, CT>(x[0], x[1]);
            *(uint4*)(at + (((gr * 2 + 1) ^ kmajor_swz<128>(ch)) << 4)) = widen_here<DT, CT>(x[2], x[3]);
        }
    };
    auto put_scales = [&](int ck) __attribute__((always_inline)) {
        if (tid < 4) {
            const float v = __builtin_fmaxf(vs, 0x1p-100f);
            f32x4 s4 = {sc * ks, __builtin_amdgcn_logf(v), __builtin_amdgcn_rcpf(v), 0.f};
            if (!sok) s4 = f32x4{0.f, -__builtin_inff(), 1.f, 0.f};      // not there: no weight
            *(f32x4*)(lds_s + (ck & 3) * 64 + tid * 16) = s4;
        }
    };
    auto barrier = []() __attribute__((always_inline)) { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

    fetch_ids(c0, c0);
    fetch(c0, c0);
    uint4 qf[KSTEPS];
    {
        const unsigned flip = p.scale_log2e < 0.f ? 0x80008000u : 0u;
        const char* const q = (const char*)p.Q + 2 * (b * p.q_bs + t_lane * p.q_rs + (long long)(h * p.G + g_lane) * p.q_hs);
#pragma unroll
        for (int k = 0; k < KSTEPS; ++k) {
            qf[k] = live ? *(const uint4*)(q + k * 32 + g * 16) : make_uint4(0, 0, 0, 0);
            qf[k] = make_uint4(qf[k].x ^ flip, qf[k].y ^ flip, qf[k].z ^ flip, qf[k].w ^ flip);
        }
    }
    fetch_ids(c0 + 1, c0);
#pragma unroll
    for (int u = 0; u < U; ++u) put_unit(u, c0, c0);
    put_scales(c0);
    fetch(c0 + 1, c0);                               // (the values of the first chunk again, which are there: the same store twice)
    fetch_ids(c0 + 2, c0 + 1);
#pragma unroll
    for (int u = 0; u < U; ++u) put_unit(u, c0 + 1, c0);
    put_scales(c0 + 1);
    fetch(c0 + 2, c0 + 1);
    fetch_ids(c0 + 3, c0 + 2);

    f32x16 acc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] = 0.f;
    float m_run = -__FLT_MAX__, l_run = 0.f;
    const int krow = 16 * ((l31 >> 2) & 1) + 4 * (l31 >> 3) + (l31 & 3);
    const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

    auto k_frag = [&](int i, int t) __attribute__((always_inline)) -> uint4 {      // product t of K Q^T: k-step t / 2, keys 32 * (t % 2) ..
        const int k = t >> 1;
        return *(const uint4*)(smem + (i & 1) * KBYTES + (k >> 2) * (64 * 128) + ((t & 1) * 32 + krow) * 128 + ((((k & 3) * 2 + g) ^ swz_k(krow)) << 4));
    };
    auto v_frag = [&](int i, int t) __attribute__((always_inline)) -> uint4 {      // product t of V^T P^T: keys of step t / DB, channels 32 * (t % DB) ..
        const int jb = t / (2 * DB), ss = t / DB % 2;
        return *(const uint4*)(lds_v + (i & 1) * VBYTES + (t % DB * 32 + l31) * 128 + (((jb * 4 + 2 * g + ss) ^ kmajor_swz<128>(l31)) << 4));
    };
    auto scales = [&](int i, int jb) __attribute__((always_inline)) -> f32x4 { return *(const f32x4*)(lds_s + (i & 3) * 64 + (jb * 2 + g) * 16); };
    auto mask = [&](int i, f32x16 (&s)[2]) __attribute__((always_inline)) {
        if (i * 64 + 64 > wmin) {
#pragma unroll
            for (int jb = 0; jb < 2; ++jb) {
                const int n = lim - i * 64 - jb * 32 - 16 * g;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[jb][r] = r < n ? s[jb][r] : -__builtin_inff();
            }
        }
    };
    // The largest t = s * factor + log2(vs) of the row in a chunk, from the scores' maxima (a factor of zero times a masked score is NaN, which a maximum passes over).
    auto raise = [&](int i, float m0, float m1) __attribute__((always_inline)) {
        const f32x4 a = scales(i, 0), c = scales(i, 1);
        float mx = __builtin_fmaxf(__builtin_fmaf(m0, a[0], a[1]), __builtin_fmaf(m1, c[0], c[1]));
        mx = __builtin_fmaxf(half_max(mx), -__FLT_MAX__);
        if (__builtin_amdgcn_ballot_w64(mx > m_run) != 0) {
            const float m_new = __builtin_fmaxf(m_run, mx);
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[db][r] *= alpha;
        }
    };

    constexpr int NQK = 2 * KSTEPS, NPV = 4 * DB, EPM = 32 / NQK;      // products; exponentials per product of the first kind
    constexpr int LAK = DH == 64 ? 4 : 2, LAV = DH == 64 ? 3 : 2;      // products by which an operand's read runs ahead
    // Chunk i: its scores are in cur and m_run is its reference.
    auto chunk_step = [&](int i, f32x16 (&cur)[2], f32x16 (&nxt)[2], auto last_flag) __attribute__((always_inline)) {
        constexpr bool LAST = decltype(last_flag)::value;
        const float ref = m_run - weight_bits<DT>();
        float mul[2], base[2], inv_vs[2];
#pragma unroll
        for (int jb = 0; jb < 2; ++jb) {
            const f32x4 s4 = scales(i, jb);
            mul[jb] = s4[0];
            base[jb] = s4[1] - ref;
            inv_vs[jb] = s4[2];
        }
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(__builtin_fabsf(m_run) <= 1024.f) || mul[0] == 0.f || mul[1] == 0.f) != 0, 0)) {
#pragma clang fp contract(off)
            // exponents in place of the scores: for references beyond 1024 the rounding of a reference alone would be seen, and a factor of zero leaves masked scores NaN
#pragma unroll
            for (int jb = 0; jb < 2; ++jb) {
                const float lvs = scales(i, jb)[1];
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float t = __builtin_fmaf(cur[jb][r], mul[jb], lvs) - ref;
                    cur[jb][r] = cur[jb][r] == -__builtin_inff() ? cur[jb][r] : t;
                }
                mul[jb] = 1.f;
                base[jb] = 0.f;
            }
        }
        unsigned pw[16];
        float lsum[2] = {0.f, 0.f};
        uint4 kf[LAK], vf[LAV];
        if constexpr (!LAST) {
#pragma unroll
            for (int t = 0; t < LAK; ++t) kf[t] = k_frag(i + 1, t);
        }
        TIR_FENCE();
#pragma unroll
        for (int t = 0; t < NQK; ++t) {
            if constexpr (!LAST) {
                nxt[t & 1] = InTraits<DT>::mfma(kf[t % LAK], qf[t >> 1], t < 2 ? zero16 : nxt[t & 1]);
                TIR_FENCE();
                if (t + LAK < NQK) kf[t % LAK] = k_frag(i + 1, t + LAK);
                // keys of chunk i + 2 and values of chunk i + 1 to LDS, then the next ones on their way
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (t == 1 + u * (NQK - 4) / U) put_unit(u, i + 2, i + 1);
                if (t == NQK - 4) put_scales(i + 2);
                if (t == NQK - 3) fetch(i + 3, i + 2);
                if (t == NQK - 2) fetch_ids(i + 4, i + 3);
            }
            if (t >= NQK - LAV) vf[t - (NQK - LAV)] = v_frag(i, t - (NQK - LAV));
#pragma unroll
            for (int e = t * EPM; e < (t + 1) * EPM; e += 2) {
                const int jb = e / 16, r = e % 16;
                float x[2];
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    x[z] = __builtin_amdgcn_exp2f(__builtin_fmaf(cur[jb][r + z], mul[jb], base[jb]));
                    lsum[jb] += x[z];
                }
                pw[e / 2] = pack2<DT>(x[0], x[1]);
            }
            TIR_FENCE();
        }
        l_run = __builtin_fmaf(lsum[0], inv_vs[0], __builtin_fmaf(lsum[1], inv_vs[1], l_run));
        if constexpr (!LAST) mask(i + 1, nxt);
        float mx[4];
#pragma unroll
        for (int t = 0; t < NPV; ++t) {
            const int at = t / DB * 4;               // keys 16*(t / DB) .. of each half-wave's order: registers of pw
            acc[t % DB] = InTraits<DT>::mfma(vf[t % LAV], make_uint4(pw[at], pw[at + 1], pw[at + 2], pw[at + 3]), acc[t % DB]);
            TIR_FENCE();
            if (t + LAV < NPV) vf[t % LAV] = v_frag(i, t + LAV);
            if constexpr (!LAST) {
                // the largest of chunk i + 1's scores, per granule, from the second product on: mx[jb], mx[2 + jb]
                constexpr int PER = (32 + NPV - 2) / (NPV - 1);
#pragma unroll
                for (int e = (t - 1) * PER; t > 0 && e < t * PER && e < 32; ++e) {
                    const int jb = e & 1, r = e >> 1, k = jb + 2 * (r & 1);
                    mx[k] = r < 2 ? nxt[jb][r] : __builtin_fmaxf(mx[k], nxt[jb][r]);
                }
            }
            TIR_FENCE();
        }
        if constexpr (!LAST) raise(i + 1, __builtin_fmaxf(mx[0], mx[2]), __builtin_fmaxf(mx[1], mx[3]));
    };

    f32x16 s_even[2], s_odd[2];
    if (c0 < c1) {
        barrier();
#pragma unroll
        for (int t = 0; t < NQK; ++t) s_even[t & 1] = InTraits<DT>::mfma(k_frag(c0, t), qf[t >> 1], t < 2 ? zero16 : s_even[t & 1]);
        mask(c0, s_even);
        float m[2];
#pragma unroll
        for (int jb = 0; jb < 2; ++jb) {
            m[jb] = s_even[jb][0];
#pragma unroll
            for (int r = 1; r < 16; ++r) m[jb] = __builtin_fmaxf(m[jb], s_even[jb][r]);
        }
        raise(c0, m[0], m[1]);
        barrier();                                   // (the first chunk's keys are overwritten from here on)
        int i = c0;
        for (; i + 2 < c1; i += 2) {
            chunk_step(i, s_even, s_odd, std::false_type());
            barrier();
            chunk_step(i + 1, s_odd, s_even, std::false_type());
            barrier();
        }
        if (i + 1 < c1) {
            chunk_step(i, s_even, s_odd, std::false_type());
            barrier();
            ++i;
#pragma unroll
            for (int jb = 0; jb < 2; ++jb) s_even[jb] = s_odd[jb];
        }
        chunk_step(i, s_even, s_odd, std::true_type());
    }
    const float l = l_run + __shfl_xor(l_run, 32);
    if (share.active > 1) {                          // partial results, joined by cache_join_kernel: [tile][slice][wave] as the other kernel's
        char* const o = (char*)p.ws + (((long long)blockIdx.x * p.slices + blockIdx.y) * QW + wave) * cache_partial_bytes<DH>();
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4) ((f32x4*)o)[(db * 4 + q4) * 64 + lane] = f32x4{acc[db][4 * q4], acc[db][4 * q4 + 1], acc[db][4 * q4 + 2], acc[db][4 * q4 + 3]};
        ((float*)(o + DB * 4096))[lane] = l;
        ((float*)(o + DB * 4096))[64 + lane] = m_run;
        return;
    }
    if (!live) return;
    const float inv = lim > 0 && l != 0.f ? 1.0f / l : 0.f;
    const long long at = b * p.o_bs + t_lane * p.o_rs + (long long)(h * p.G + g_lane) * p.o_hs;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
            const int ch = db * 32 + q4 * 8 + 4 * g;
            const f32x4 v = {acc[db][4 * q4] * inv, acc[db][4 * q4 + 1] * inv, acc[db][4 * q4 + 2] * inv, acc[db][4 * q4 + 3] * inv};
            if (p.out32) *(f32x4*)((float*)p.O + at + ch) = v;
            else *(uint2*)((unsigned short*)p.O + at + ch) = make_uint2(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]));
        }
}

// Joins the slices of cache_tile_kernel, in slice order: a workgroup per wave of a tile, one thread for a quarter of the channels of a row's half.
template <int DT, int DH, int QW> __global__ void __launch_bounds__(256) cache_join_kernel(const CacheAttnParams p) {
    constexpr int DB = DH / 32, PART = cache_partial_bytes<DH>();
    const int tile = (int)blockIdx.x, wave = (int)blockIdx.y;
    const int bh = (int)fastdiv((unsigned)tile, p.div_tiles_magic, p.div_tiles_shift);
    const int row0 = (tile - bh * p.tiles) * (QW * 32);
    const int b = (int)fastdiv((unsigned)bh, p.div_h_magic, p.div_h_shift), h = bh - b * p.c.heads;
    const long long cap = (long long)p.c.cols << p.c.shift;
    int len = p.lens[b], cnt = p.count ? p.count[b] : p.T;
    len = len < 0 ? 0 : (len > (int)cap ? (int)cap : len);
    cnt = cnt < 0 ? 0 : (cnt > p.T ? p.T : cnt);
    const int rows = cnt * p.G - row0;
    if (rows <= wave * 32) return;
    const int last = row0 + (rows < QW * 32 ? rows : QW * 32) - 1;
    const long long kmax = (long long)len - cnt + (int)fastdiv((unsigned)last, p.div_g_magic, p.div_g_shift) + 1;
    const int active = tile_share(kmax < 0 ? 0 : (int)kmax, p.slices).active;
    if (active == 1) return;
    const int lane = (int)threadIdx.x & 63, l31 = lane & 31, g = lane >> 5, db = (int)threadIdx.x >> 6;
    if (db >= DB) return;
    const char* const part = (const char*)p.ws + ((long long)tile * p.slices * QW + wave) * PART;
    auto slice = [&](int z) { return part + (long long)z * QW * PART; };
    float top = -__FLT_MAX__, l = 0.f;
#pragma unroll 4
    for (int z = 0; z < active; ++z) top = __builtin_fmaxf(top, ((const float*)(slice(z) + DB * 4096))[64 + lane]);
    f32x4 out[4];
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) out[q4] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int z = 0; z < active; ++z) {
        const float f = __builtin_amdgcn_exp2f(((const float*)(slice(z) + DB * 4096))[64 + lane] - top);
        l += f * ((const float*)(slice(z) + DB * 4096))[lane];
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) out[q4] += f * ((const f32x4*)slice(z))[(db * 4 + q4) * 64 + lane];
    }
    if (wave * 32 + l31 >= rows) return;
    const int row = row0 + wave * 32 + l31;
    const int t = (int)fastdiv((unsigned)row, p.div_g_magic, p.div_g_shift);
    const bool seen = (long long)len - cnt + t + 1 > 0;
    const float inv = seen && l != 0.f ? 1.0f / l : 0.f;
    const long long at = b * p.o_bs + t * p.o_rs + (long long)(h * p.G + row - t * p.G) * p.o_hs + db * 32 + 4 * g;
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
        const f32x4 v = out[q4] * inv;
        if (p.out32) *(f32x4*)((float*)p.O + at + q4 * 8) = v;
        else *(uint2*)((unsigned short*)p.O + at + q4 * 8) = make_uint2(pack2<DT>(v[0], v[1]), pack2<DT>(v[2], v[3]));
    }
}

}  // namespace tir
