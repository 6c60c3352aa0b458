// Gradients of the attention over another sequence's states: entry point, split of the work, launches.
#include <stdint.h>

#include "tir_cross_grad.h"
#include "tir_host.h"
#include "tir_launch.h"

namespace tir {

// Two groups of waves on a tile's keys where there is one workgroup per CU.
static int keys_pass_groups(int64_t tiles, int64_t slices) { return tiles * slices <= 256 ? 2 : 1; }

template <int DT, int DH, bool TWO> static hipError_t launch_rows_pass(const GradParams& p, dim3 grid, hipStream_t stream) {
    return launch_kernel(p.N <= kFewKeys ? &grad_rows_kernel<DT, DH, true, TWO> : &grad_rows_kernel<DT, DH, false, TWO>, grid, dim3(kGradThreads), stream, p);
}
template <int DT, int DH, bool KEYS> static hipError_t launch_pass(const GradParams& p, bool two, hipStream_t stream) {
    const unsigned tiles = (unsigned)(p.batch * p.heads * p.tiles);
    const dim3 grid(tiles, (unsigned)p.slices);
    hipError_t e;
    if (!KEYS) e = two ? launch_rows_pass<DT, DH, true>(p, grid, stream) : launch_rows_pass<DT, DH, false>(p, grid, stream);
    else if (two) e = launch_kernel(&grad_keys_kernel<DT, DH, 2, true>, grid, dim3(2 * kGradThreads), stream, p);
    else if (keys_pass_groups(tiles, p.slices) == 2) e = launch_kernel(&grad_keys_kernel<DT, DH, 2, false>, grid, dim3(2 * kGradThreads), stream, p);
    else e = launch_kernel(&grad_keys_kernel<DT, DH, 1, false>, grid, dim3(kGradThreads), stream, p);
    if (e != hipSuccess || p.slices == 1) return e;
    return launch_kernel(&grad_sum_kernel<DT, DH, KEYS>, dim3((KEYS ? 2 : 1) * kGradTile * DH / 1024, tiles), dim3(256), stream, p);
}
template <bool KEYS> static hipError_t launch_by_type(const GradParams& p, int dt, int dh, bool two, hipStream_t stream) {
    if (dt == DT_F16 && dh == 64) return launch_pass<DT_F16, 64, KEYS>(p, two, stream);
    if (dt == DT_F16 && dh == 128) return launch_pass<DT_F16, 128, KEYS>(p, two, stream);
    if (dt == DT_BF16 && dh == 64) return launch_pass<DT_BF16, 64, KEYS>(p, two, stream);
    if (dt == DT_BF16 && dh == 128) return launch_pass<DT_BF16, 128, KEYS>(p, two, stream);
    return hipErrorInvalidValue;
}
hipError_t launch_grad_rows(const GradParams& p, int dt, int dh, bool two, hipStream_t stream) { return launch_by_type<false>(p, dt, dh, two, stream); }
hipError_t launch_grad_keys(const GradParams& p, int dt, int dh, bool two, hipStream_t stream) { return launch_by_type<true>(p, dt, dh, two, stream); }

// How many workgroups share a tile's walk of `steps` chunks (of 64 rows or keys): as many as the chip has room for, each with two chunks at least, as far as the partial sums fit.
static int slices_of(int64_t tiles, int64_t room, int64_t steps, int64_t part_bytes, const StreamWorkspace& ws) {
    if (!ws.partial || tiles >= room) return 1;
    int64_t s = room / tiles;
    if (s > steps / 2) s = steps / 2;
    if (s > ws.bytes / (tiles * part_bytes)) s = ws.bytes / (tiles * part_bytes);
    return s > 64 ? 64 : s < 2 ? 1 : (int)s;
}

}  // namespace tir

using namespace tir;

extern "C" {

tir_status tir_cross_attention_backward(const void* Q, const void* K, const void* V, const void* O, const void* dO,
                                        const float* lse, const int32_t* lens, void* dQ, void* dK, void* dV,
                                        float* delta, int64_t batch, int64_t M, int64_t N, int64_t Hq, int64_t Hkv,
                                        int64_t d, int64_t q_bs, int64_t q_rs, int64_t q_hs, int64_t k_bs,
                                        int64_t k_rs, int64_t k_hs, int64_t v_bs, int64_t v_rs, int64_t v_hs,
                                        int64_t o_bs, int64_t o_rs, int64_t o_hs, int64_t g_bs, int64_t g_rs,
                                        int64_t g_hs, float scale, tir_dtype in, tir_stream stream) {
    const char* const who = "cross attention backward";
    if ((int)in < 0 || (int)in > TIR_E4M3) return host_error(TIR_ERR_INVALID_ARG, "unknown dtype code (in=%d)", (int)in);
    if (in != TIR_F16 && in != TIR_BF16) return host_error(TIR_ERR_UNSUPPORTED, "%s: unsupported dtype %d", who, (int)in);
    tir_status st = check_cross(who, batch, M, N, Hq, Hkv, d, scale);
    if (st == TIR_OK) st = check_row_strides(who, "Q", q_bs, q_rs, q_hs);
    if (st == TIR_OK) st = check_row_strides(who, "K", k_bs, k_rs, k_hs);
    if (st == TIR_OK) st = check_row_strides(who, "V", v_bs, v_rs, v_hs);
    if (st == TIR_OK) st = check_row_strides(who, "O", o_bs, o_rs, o_hs);
    if (st == TIR_OK) st = check_row_strides(who, "dO", g_bs, g_rs, g_hs);
    if (st != TIR_OK) return st;
    if (batch == 0 || Hq == 0) return TIR_OK;
    if ((batch > 1 && q_bs == 0) || (M > 1 && q_rs == 0) || (Hq > 1 && q_hs == 0)) return host_error(TIR_ERR_INVALID_ARG, "%s: a stride of Q is zero: the gradients of its rows overlap", who);
    if ((batch > 1 && (k_bs == 0 || v_bs == 0)) || (N > 1 && (k_rs == 0 || v_rs == 0)) || (Hkv > 1 && (k_hs == 0 || v_hs == 0)))
        return host_error(TIR_ERR_INVALID_ARG, "%s: a stride of K or V is zero: the gradients of their rows overlap", who);
    if (M > 0 && (!Q || !O || !dO || !lse || !dQ || !delta)) return host_error(TIR_ERR_INVALID_ARG, "%s: Q, O, dO, lse, dQ or delta is null", who);
    if (N > 0 && (!K || !V || !dK || !dV)) return host_error(TIR_ERR_INVALID_ARG, "%s: K, V, dK or dV is null", who);
    const void* const wide[] = {Q, K, V, O, dO, dQ, dK, dV};
    for (const void* x : wide)
        if (!host_aligned(x, 16)) return host_error(TIR_ERR_ALIGNMENT, "%s: the tensors must be 16-byte aligned", who);
    if (!host_aligned(lse, 4) || !host_aligned(delta, 4) || !host_aligned(lens, 4)) return host_error(TIR_ERR_ALIGNMENT, "%s: lse, delta and lens must be 4-byte aligned", who);
    GradParams p = {};
    p.Q = Q; p.K = K; p.V = V; p.O = O; p.dO = dO;
    p.dQ = dQ; p.dK = dK; p.dV = dV;
    p.lse = lse; p.delta = delta; p.lens = lens;
    p.q_bs = q_bs; p.q_rs = q_rs; p.q_hs = q_hs;
    p.k_bs = k_bs; p.k_rs = k_rs; p.k_hs = k_hs;
    p.v_bs = v_bs; p.v_rs = v_rs; p.v_hs = v_hs;
    p.o_bs = o_bs; p.o_rs = o_rs; p.o_hs = o_hs;
    p.g_bs = g_bs; p.g_rs = g_rs; p.g_hs = g_hs;
    p.M = (int)M; p.N = (int)N;
    p.heads = (int)Hkv;
    p.G = (int)(Hq / Hkv);
    p.batch = (int)batch;
    p.scale = scale;
    p.q_near = q_rs < (1 << 20) && q_hs < (1 << 28) / p.G;      // a tile's 128 rows: at most 127 * q_rs * 2 + (G - 1) * q_hs * 2 bytes
    p.scale_log2e = scale * 1.44269504088896340736f;
    const FastDiv dh = make_fastdiv((unsigned)p.heads), dg = make_fastdiv((unsigned)p.G);
    p.div_h_magic = dh.magic; p.div_h_shift = dh.shift;
    p.div_g_magic = dg.magic; p.div_g_shift = dg.shift;
    const StreamWorkspace ws = stream_workspace((hipStream_t)stream);
    p.ws = (float*)ws.partial;
    const int64_t row_tiles = (M * p.G + kGradTile - 1) / kGradTile, key_tiles = (N + kGradTile - 1) / kGradTile;
    // (before the passes are planned: slices that share a tile's rows stay within 256 workgroups)
    const bool two = (double)batch * Hq * M * N <= kTwoParts && keys_pass_groups(batch * Hkv * key_tiles, 1) == 2;
    auto pass = [&](bool keys, int64_t tiles, int64_t steps) {
        const FastDiv dt = make_fastdiv((unsigned)tiles);
        p.tiles = (int)tiles;
        p.div_tiles_magic = dt.magic; p.div_tiles_shift = dt.shift;
        p.slices = slices_of(batch * Hkv * tiles, keys ? 256 : 512, steps, 4 * grad_partial(keys, (int)d), ws);
        return keys ? launch_grad_keys(p, (int)in, (int)d, two, (hipStream_t)stream) : launch_grad_rows(p, (int)in, (int)d, two, (hipStream_t)stream);
    };
    if (!grid_fits(batch * Hkv * row_tiles, kGradThreads) || !grid_fits(batch * Hkv * key_tiles, kGradThreads)) return launch_error(who, hipErrorInvalidConfiguration);
    hipError_t e = hipSuccess;
    if (M > 0) e = pass(false, row_tiles, (N + 63) / 64);
    if (e == hipSuccess && N > 0) e = pass(true, key_tiles, (M + 63) / 64 * p.G);
    if (e != hipSuccess) return launch_error(who, e);
    return TIR_OK;
}

}  // extern "C"
