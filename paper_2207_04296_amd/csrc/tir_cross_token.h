// Attention of a few rows of a key head - a single token's query heads - over another sequence's states.
//
// No tile of the matrix intrinsic: of its 32 (16) columns one to four would be used, and its operand V^T has to be transposed through LDS.  Here LPK lanes share a key, eight channels each, in
// 16-byte loads straight into registers; a score is a sum of two-element dot products and an exchange between those lanes, the output eight multiply-adds per key and lane.  Every group of LPK lanes runs
// the softmax over its own keys, and groups, waves and slices are joined at the end.  Probabilities are not rounded.
// Bound by memory: 2 * 16 bytes per lane and 26 vector instructions per row, of a budget of about 80 at the rate the chip's memory delivers.
#pragma once
#include "tir_attention.h"

namespace tir {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int kTokenWaves = 4, kTokenRows = 4;      // most rows of a call

template <int DT> __device__ __forceinline__ float dot2(unsigned a, unsigned b, float c) {
    if constexpr (DT == DT_F16) {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, a), __builtin_bit_cast(h2, b), c, false);
    } else {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b2, a), __builtin_bit_cast(b2, b), c, false);
    }
}
template <int DT, int I> __device__ __forceinline__ float half_of(unsigned w) {      // its low (0) or high (1) value
    if constexpr (DT == DT_F16) {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        return (float)__builtin_bit_cast(h2, w)[I];
    } else {
        return __builtin_bit_cast(float, I ? w & 0xffff0000u : w << 16);
    }
}

template <int CTRL> __device__ __forceinline__ float add_dpp(float x) {
    const int y = __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true);
    return x + __builtin_bit_cast(float, y);
}
// Sum over the 8 or 16 consecutive lanes of a key, in all of them: neighbours, pairs, and once these agree the mirror images of 8 and 16 lanes.  (Data-parallel moves inside the additions:
// through LDS permutes 4 rows of 128 channels over 100 000 keys took 125 us, 91.5 this way.)
template <int N> __device__ __forceinline__ float sum_lanes(float x) {
    x = add_dpp<0xB1>(x);       // quad_perm [1,0,3,2]
    x = add_dpp<0x4E>(x);       // quad_perm [2,3,0,1]
    x = add_dpp<0x141>(x);      // row_half_mirror
    if constexpr (N == 16) x = add_dpp<0x140>(x);      // row_mirror
    return x;
}

// Partial results of a slice: per row DH sums, the sum of probabilities, the reference.
template <int DH> constexpr int cross_token_partial(int rows) { return rows * (DH + 2) * 4; }

// R: rows of a (sequence, key head).  Keys of a chunk: four loads of 64 / LPK keys.
template <int DT, int DH, int R>
__global__ void __launch_bounds__(kTokenWaves * 64) cross_token_kernel(const CrossParams p) {
    constexpr int LPK = DH / 8, KPL = 64 / LPK, NL = 4, CK = NL * KPL, KG = kTokenWaves;
    __shared__ float smem[KG][R][DH + 2];
    __shared__ unsigned arrived;
    const int lane = threadIdx.x & 63, sub = lane & (LPK - 1), key_of = lane / LPK;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = (int)blockIdx.x;
    const int seq = (int)fastdiv((unsigned)tile, p.div_h_magic, p.div_h_shift);
    const int head = tile - seq * p.heads;
    int n = p.N;
    if (p.lens) {
        n = p.lens[seq];
        n = n < 0 ? 0 : (n > p.N ? p.N : n);
    }
    const int nch = (n + CK - 1) / CK;
    int per = (nch + p.slices - 1) / p.slices;
    per = (per + KG - 1) / KG * KG;
    const int active = nch > per ? (nch + per - 1) / per : 1;
    if ((int)blockIdx.y >= active) return;
    const int c_end = ((int)blockIdx.y + 1) * per < nch ? ((int)blockIdx.y + 1) * per : nch;
    const int c_first = (int)blockIdx.y * per + wave;
    const int mine = c_end > c_first ? (c_end - c_first + KG - 1) / KG : 0;

    const char* const Kb = (const char*)p.K + 2 * (seq * p.k_bs + head * p.k_hs) + sub * 16;
    const char* const Vb = (const char*)p.V + 2 * (seq * p.v_bs + head * p.v_hs) + sub * 16;
    const unsigned k_rs = (unsigned)p.k_rs * 2, v_rs = (unsigned)p.v_rs * 2;
    auto place = [&](int r, long long bs, long long rs, long long hs) __attribute__((always_inline)) -> long long {
        const int m = (int)fastdiv((unsigned)r, p.div_g_magic, p.div_g_shift);
        return seq * bs + m * rs + (long long)(head * p.G + r - m * p.G) * hs;
    };
    struct Chunk {
        u32x4 k[NL], v[NL];
    };
    auto load = [&](int i, Chunk& c) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NL; ++u) {
            const int key = (c_first + i * KG) * CK + u * KPL + key_of;
            const unsigned at = (unsigned)(key < n ? key : n - 1);      // (one that is there again where there is none: it gets no weight, and step clears its value)
            c.k[u] = *(const u32x4*)(Kb + (unsigned long long)at * k_rs);
            c.v[u] = *(const u32x4*)(Vb + (unsigned long long)at * v_rs);
        }
    };
    Chunk even, odd;
    if (mine > 0) load(0, even);
    u32x4 q[R];
#pragma unroll
    for (int r = 0; r < R; ++r) q[r] = *(const u32x4*)((const char*)p.Q + 2 * place(r, p.q_bs, p.q_rs, p.q_hs) + sub * 16);
    float acc[R][8], m_run[R], l_run[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        m_run[r] = -__FLT_MAX__;
        l_run[r] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[r][e] = 0.f;
    }
    auto step = [&](int i, Chunk& c) __attribute__((always_inline)) {
        const int left = n - (c_first + i * KG) * CK - key_of;      // load u has a key of this lane's if u * KPL < left
        if ((c_first + i * KG + 1) * CK > n) {                      // (an infinite or NaN value times a weight of zero is NaN)
#pragma unroll
            for (int u = 0; u < NL; ++u)
                if (u * KPL >= left) c.v[u] = u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float t[NL];
#pragma unroll
            for (int u = 0; u < NL; ++u) {
                float s = 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) s = dot2<DT>(q[r][e], c.k[u][e], s);
                t[u] = u * KPL < left ? sum_lanes<LPK>(s) * p.scale_log2e : -__builtin_inff();
            }
            float mx = t[0];
#pragma unroll
            for (int u = 1; u < NL; ++u) mx = __builtin_fmaxf(mx, t[u]);
            mx = __builtin_fmaxf(mx, m_run[r]);
            const float alpha = __builtin_amdgcn_exp2f(m_run[r] - mx);
            m_run[r] = mx;
            l_run[r] *= alpha;
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[r][e] *= alpha;
#pragma unroll
            for (int u = 0; u < NL; ++u) {
                const float w = __builtin_amdgcn_exp2f(t[u] - mx);
                l_run[r] += w;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    acc[r][2 * e] = __builtin_fmaf(w, half_of<DT, 0>(c.v[u][e]), acc[r][2 * e]);
                    acc[r][2 * e + 1] = __builtin_fmaf(w, half_of<DT, 1>(c.v[u][e]), acc[r][2 * e + 1]);
                }
            }
        }
    };
    for (int i = 0; i < mine; i += 2) {
        load(i + 1, odd);                            // (behind the last chunk: the last key again)
        step(i, even);
        load(i + 2, even);
        if (i + 1 < mine) step(i + 1, odd);
    }

    // ------------------------------------------------------------ the groups of lanes, then the waves
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float top = m_run[r];
#pragma unroll
        for (int x = LPK; x < 64; x <<= 1) top = __builtin_fmaxf(top, __shfl_xor(top, x));
        const float f = __builtin_amdgcn_exp2f(m_run[r] - top);
        float l = l_run[r] * f;
#pragma unroll
        for (int x = LPK; x < 64; x <<= 1) l += __shfl_xor(l, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float a = acc[r][e] * f;
#pragma unroll
            for (int x = LPK; x < 64; x <<= 1) a += __shfl_xor(a, x);
            if (key_of == 0) smem[wave][r][sub * 8 + e] = a;
        }
        if (lane == 0) {
            smem[wave][r][DH] = l;
            smem[wave][r][DH + 1] = top;
        }
    }
    __syncthreads();
    constexpr int OUTS = R * DH, PER = (OUTS + KG * 64 - 1) / (KG * 64);      // values per thread
    float out[PER], l[PER], top[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int x = (int)threadIdx.x + i * KG * 64, r = x / DH, ch = x % DH;
        out[i] = l[i] = 0.f;
        top[i] = -__FLT_MAX__;
        if (x < OUTS) {
#pragma unroll
            for (int k = 0; k < KG; ++k) top[i] = __builtin_fmaxf(top[i], smem[k][r][DH + 1]);
#pragma unroll
            for (int k = 0; k < KG; ++k) {
                const float f = __builtin_amdgcn_exp2f(smem[k][r][DH + 1] - top[i]);
                out[i] += f * smem[k][r][ch];
                l[i] += f * smem[k][r][DH];
            }
        }
    }
    if (active > 1) {
        // As in the split reductions: partial results at system scope, the last to arrive adds them in slice order.
        constexpr int kSystemScope = 17, PART = cross_token_partial<DH>(R);
        const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc((char*)p.ws + (long long)tile * p.slices * PART, 0, p.slices * PART, 0x00020000);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int x = (int)threadIdx.x + i * KG * 64, r = x / DH, ch = x % DH;
            if (x < OUTS) {
                __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, out[i]), rw, (r * (DH + 2) + ch) * 4, (int)blockIdx.y * PART, kSystemScope);
                if (ch == 0) {
                    __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, l[i]), rw, (r * (DH + 2) + DH) * 4, (int)blockIdx.y * PART, kSystemScope);
                    __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, top[i]), rw, (r * (DH + 2) + DH + 1) * 4, (int)blockIdx.y * PART, kSystemScope);
                }
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) arrived = __hip_atomic_fetch_add(p.ws_count + tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
        __syncthreads();
        if (arrived != (unsigned)active - 1u) return;
        if (threadIdx.x == 0) __hip_atomic_store(p.ws_count + tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            out[i] = l[i] = 0.f;
            top[i] = -__FLT_MAX__;
        }
        constexpr int Z = 8;                         // slices on their way at a time
        for (int z0 = 0; z0 < active; z0 += Z) {
            float a[PER][Z], b[PER][Z], m[PER][Z];
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int x = (int)threadIdx.x + i * KG * 64, r = x / DH, ch = x % DH;
#pragma unroll
                for (int z = 0; z < Z; ++z) {
                    const int row = z0 + z < active && x < OUTS ? r * (DH + 2) * 4 : (int)kOutOfRange;
                    a[i][z] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rw, row + ch * 4, (z0 + z) * PART, kSystemScope));
                    b[i][z] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rw, row + DH * 4, (z0 + z) * PART, kSystemScope));
                    m[i][z] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rw, row + (DH + 1) * 4, (z0 + z) * PART, kSystemScope));
                }
            }
#pragma unroll
            for (int i = 0; i < PER; ++i)
#pragma unroll
                for (int z = 0; z < Z; ++z) {
                    if (z0 + z < active) {
                        const float mx = __builtin_fmaxf(top[i], m[i][z]), fo = __builtin_amdgcn_exp2f(top[i] - mx), fn = __builtin_amdgcn_exp2f(m[i][z] - mx);
                        top[i] = mx;
                        out[i] = out[i] * fo + a[i][z] * fn;
                        l[i] = l[i] * fo + b[i][z] * fn;
                    }
                }
        }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int x = (int)threadIdx.x + i * KG * 64, r = x / DH, ch = x % DH;
        if (x < OUTS) {
            const float o = n > 0 ? out[i] / l[i] : 0.f;
            const long long at = place(r, p.o_bs, p.o_rs, p.o_hs) + ch;
            if (p.out32) ((float*)p.O)[at] = o;
            else ((typename OutTraits<DT>::type*)p.O)[at] = OutTraits<DT>::cvt(o);
            if (ch == 0 && p.lse) {
                const int m = (int)fastdiv((unsigned)r, p.div_g_magic, p.div_g_shift);
                p.lse[((long long)seq * p.heads * p.G + head * p.G + r - m * p.G) * p.positions + m] = n > 0 ? (top[i] + __builtin_amdgcn_logf(l[i])) * 0.69314718055994530942f : -__builtin_inff();
            }
        }
    }
}

hipError_t launch_cross_token(const CrossParams& p, int dt, int dh, hipStream_t stream);

}  // namespace tir
