// Attention over the states of another sequence (forward): entry point, choice of kernel, instantiations of the attention kernel for strided
// operands.
#include <stdint.h>

#include "tir_attention.h"
#include "tir_cross_token.h"
#include "tir_host.h"
#include "tir_launch.h"

namespace tir {

template <int DT, int OUT, int DH, int QW, int KG, int KB, int FORM> static hipError_t launch_cross_as(CrossParams p, hipStream_t stream) {
    p.tiles_m = (p.M + 32 * QW - 1) / (32 * QW);
    const FastDiv dtm = make_fastdiv((unsigned)p.tiles_m);
    p.div_tm_magic = dtm.magic;
    p.div_tm_shift = dtm.shift;
    if (!grid_fits((int64_t)p.batch * p.tiles_m, QW * KG * 64)) return hipErrorInvalidConfiguration;
    return launch_kernel(&attention_kernel<DT, OUT, DH, QW, KG, KB, FORM, CrossParams>, dim3((unsigned)(p.batch * p.tiles_m), KG > 1 ? (unsigned)p.slices : 1u), dim3(QW * KG * 64), stream, p);
}

// The kernel by the rule for dense heads: a (sequence, key head) with the rows of all its query heads is a head of that rule, at the largest number of keys.
// Sequences of different lengths leave the CUs of the short ones early: at d = 128 two workgroups of 128 rows per CU rather than one of 256, so that a long and a short one share a CU
// (2 x 2047 x 4095 and 1365 keys x 16 heads of 128: 136 and 108 us; at d = 64, four or two per CU, 16 x 512 x 333 .. 1000 x 16 heads the same 45 us either way).
template <int DT, int OUT, int DH> static hipError_t launch_cross(const CrossParams& p, hipStream_t stream) {
    const AttnKernel k = p.slices > 1 ? ATTN_T64_GROUPS : attention_kernel_of(p.batch, p.M, p.N, DH, OUT);
    if (k == ATTN_T64_GROUPS) return launch_cross_as<DT, OUT, DH, 2, 4, DH == 64 ? 64 : 32, ATTN_PIPED>(p, stream);
    if (k == ATTN_T128_C32) return launch_cross_as<DT, OUT, DH, 4, 1, 32, ATTN_PIPED>(p, stream);
    if (k == ATTN_T128_STREAM) return launch_cross_as<DT, OUT, DH, 4, 1, 64, ATTN_PIPED_STREAM>(p, stream);
    if constexpr (DH == 64) {
        if (k == ATTN_T128_SEQUENTIAL) return launch_cross_as<DT, OUT, DH, 4, 1, 64, ATTN_SEQUENTIAL>(p, stream);
        if (k == ATTN_T256_SEQUENTIAL) return launch_cross_as<DT, OUT, DH, 8, 1, 64, ATTN_SEQUENTIAL>(p, stream);
    } else {
        if (k == ATTN_T256 && !p.lens) return launch_cross_as<DT, OUT, DH, 8, 1, 64, ATTN_PIPED>(p, stream);
    }
    return launch_cross_as<DT, OUT, DH, 4, 1, 64, ATTN_PIPED>(p, stream);
}

cross_launch_fn cross_launcher(int dt, int out, int dh) {
#define TIR_CROSS(DT, OUT, DH) \
    if (dt == DT && out == OUT && dh == DH) return &launch_cross<DT, OUT, DH>;
    TIR_CROSS(DT_F16, DT_F16, 64) TIR_CROSS(DT_F16, DT_F32, 64) TIR_CROSS(DT_F16, DT_F16, 128) TIR_CROSS(DT_F16, DT_F32, 128)
    TIR_CROSS(DT_BF16, DT_BF16, 64) TIR_CROSS(DT_BF16, DT_F32, 64) TIR_CROSS(DT_BF16, DT_BF16, 128) TIR_CROSS(DT_BF16, DT_F32, 128)
#undef TIR_CROSS
    return nullptr;
}

}  // namespace tir

using namespace tir;

extern "C" {

tir_status tir_cross_attention(const void* Q, const void* K, const void* V, void* O, float* lse, const int32_t* lens,
                               int64_t batch, int64_t M, int64_t N, int64_t Hq, int64_t Hkv, int64_t d, int64_t q_bs,
                               int64_t q_rs, int64_t q_hs, int64_t k_bs, int64_t k_rs, int64_t k_hs, int64_t v_bs,
                               int64_t v_rs, int64_t v_hs, int64_t o_bs, int64_t o_rs, int64_t o_hs, float scale,
                               tir_dtype in, tir_dtype out, tir_stream stream) {
    const char* const who = "cross attention";
    if ((int)in < 0 || (int)in > TIR_E4M3 || (int)out < 0 || (int)out > TIR_E4M3) return host_error(TIR_ERR_INVALID_ARG, "unknown dtype code (in=%d out=%d)", (int)in, (int)out);
    if (!((in == TIR_F16 || in == TIR_BF16) && (out == in || out == TIR_F32))) return host_error(TIR_ERR_UNSUPPORTED, "%s: unsupported (in, out) dtype pair (%d, %d)", who, (int)in, (int)out);
    tir_status st = check_cross(who, batch, M, N, Hq, Hkv, d, scale);
    if (st == TIR_OK) st = check_row_strides(who, "Q", q_bs, q_rs, q_hs);
    if (st == TIR_OK) st = check_row_strides(who, "K", k_bs, k_rs, k_hs);
    if (st == TIR_OK) st = check_row_strides(who, "V", v_bs, v_rs, v_hs);
    if (st == TIR_OK) st = check_row_strides(who, "O", o_bs, o_rs, o_hs);
    if (st != TIR_OK) return st;
    if (batch == 0 || M == 0 || Hq == 0) return TIR_OK;
    if (!Q || !O || (N > 0 && (!K || !V))) return host_error(TIR_ERR_INVALID_ARG, "%s: Q, K, V or O is null", who);
    if (!host_aligned(Q, 16) || !host_aligned(K, 16) || !host_aligned(V, 16) || !host_aligned(O, 16)) return host_error(TIR_ERR_ALIGNMENT, "%s: Q, K, V and O must be 16-byte aligned", who);
    if (!host_aligned(lse, 4) || !host_aligned(lens, 4)) return host_error(TIR_ERR_ALIGNMENT, "%s: lse and lens must be 4-byte aligned", who);
    if ((batch > 1 && o_bs == 0) || (M > 1 && o_rs == 0) || (Hq > 1 && o_hs == 0)) return host_error(TIR_ERR_INVALID_ARG, "%s: a stride of O is zero: its rows overlap", who);
    cross_launch_fn fn = cross_launcher((int)in, (int)out, (int)d);
    if (!fn) return host_error(TIR_ERR_UNSUPPORTED, "%s: no kernel for this dtype pair / head dimension", who);
    CrossParams p = {};
    p.Q = Q; p.K = K; p.V = V; p.O = O;
    p.G = (int)(Hq / Hkv);
    p.positions = (int)M;
    p.M = (int)(M * p.G);
    p.N = (int)N;
    p.batch = (int)(batch * Hkv);
    p.heads = (int)Hkv;
    p.scale_log2e = scale * 1.44269504088896340736f;
    p.q_bs = q_bs; p.q_rs = q_rs; p.q_hs = q_hs;
    p.k_bs = k_bs; p.k_rs = k_rs; p.k_hs = k_hs;
    p.v_bs = v_bs; p.v_rs = v_rs; p.v_hs = v_hs;
    p.o_bs = o_bs; p.o_rs = o_rs; p.o_hs = o_hs;
    p.lens = lens;
    p.lse = lse;
    const FastDiv dh = make_fastdiv((unsigned)p.heads), dg = make_fastdiv((unsigned)p.G);
    p.div_h_magic = dh.magic; p.div_h_shift = dh.shift;
    p.div_g_magic = dg.magic; p.div_g_shift = dg.shift;
    p.out32 = out == TIR_F32;
    p.o_near = o_rs < (1 << 20) && o_hs < (1 << 28) / p.G;      // a tile's 256 rows: 255 * o_rs * 4 bytes, or with G > 1 at most 128 * o_rs * 4 + (G - 1) * o_hs * 4
    p.slices = 1;
    const StreamWorkspace ws = stream_workspace((hipStream_t)stream);
    auto share = [&](int64_t tiles, int64_t slices, int64_t most, int64_t part) {
        if (slices > most) slices = most;
        if (slices > 64) slices = 64;
        if (ws.partial && tiles <= ws.counters && slices > 1 && slices * tiles * part <= ws.bytes) {
            p.slices = (int)slices;
            p.ws = ws.partial;
            p.ws_count = ws.count;
        }
    };
    hipError_t e;
    // The vector kernel's time grows with the rows, that of a tile of 64 does not.  8 x 1500 keys x 16 heads of 64, 1, 2, 4, 5, 6 and 8 rows, us: 13.6, 14.5, 17.6, 20.7, 23.3, 28.4, and the tile 17.0 for 2 to 16;
    // x 8 heads of 128: 12.9, 13.9, 18.4, 21.3, 23.6, 28.9, and 19.0; 100 000 keys x 4 heads of 128, 4, 5 and 8 rows: 57, 70, 98, and 85.
    if (p.M <= kTokenRows && N > 0) {
        const int64_t chunk = d == 64 ? 32 : 16;         // two per wave
        share(p.batch, 256 / p.batch, N / (8 * chunk), d == 64 ? cross_token_partial<64>(p.M) : cross_token_partial<128>(p.M));
        e = launch_cross_token(p, (int)in, (int)d, (hipStream_t)stream);
        if (e != hipSuccess) return launch_error(who, e);
        return TIR_OK;
    }
    // Few tiles of 64 rows: their keys are shared among workgroups, one of which fills a CU, as long as each of its four key groups keeps two chunks.
    const int64_t tiles = (int64_t)p.batch * ((p.M + 63) / 64), chunk = d == 64 ? 64 : 32;
    if (tiles <= 128) share(tiles, 256 / tiles, N / (8 * chunk), 2 * (d / 32 * 4096 + 512));
    e = fn(p, (hipStream_t)stream);
    if (e != hipSuccess) return launch_error(who, e);
    return TIR_OK;
}

}  // extern "C"
