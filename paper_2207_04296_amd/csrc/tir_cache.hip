// Entry points of the paged cache and of attention over it: argument checks, choice of kernel, launch.
#include <stdint.h>
#include <stdio.h>

#include "tir_host.h"
#include "tir_launch.h"
#include "tir_cache.h"

namespace tir {

template <int DT, int CT, int DH> static hipError_t launch_append_as(const AppendParams& p, int64_t batch, hipStream_t stream) {
    const dim3 grid((unsigned)(batch * p.touched * p.c.heads), 2), block(kAppendThreads);
    if (!grid_fits(batch * p.touched * p.c.heads, kAppendThreads)) return hipErrorInvalidConfiguration;
    if (p.c.shift == 4) return launch_kernel(&cache_append_kernel<DT, CT, DH, 16>, grid, block, stream, p);
    if (p.c.shift == 5) return launch_kernel(&cache_append_kernel<DT, CT, DH, 32>, grid, block, stream, p);
    if (p.c.shift == 6) return launch_kernel(&cache_append_kernel<DT, CT, DH, 64>, grid, block, stream, p);
    return launch_kernel(&cache_append_kernel<DT, CT, DH, 128>, grid, block, stream, p);
}
hipError_t launch_append(const AppendParams& p, int dt, int ct, int d, int64_t batch, hipStream_t stream) {
#define TIR_APPEND(DT, CT, DH) if (dt == DT && ct == CT && d == DH) return launch_append_as<DT, CT, DH>(p, batch, stream);
    TIR_APPEND(DT_F16, CT_I8, 64) TIR_APPEND(DT_F16, CT_I8, 128) TIR_APPEND(DT_F16, CT_E4M3, 64) TIR_APPEND(DT_F16, CT_E4M3, 128)
    TIR_APPEND(DT_BF16, CT_I8, 64) TIR_APPEND(DT_BF16, CT_I8, 128) TIR_APPEND(DT_BF16, CT_E4M3, 64) TIR_APPEND(DT_BF16, CT_E4M3, 128)
#undef TIR_APPEND
    return hipErrorInvalidValue;
}

template <int DT, int CT, int DH> static hipError_t launch_cache_as(const CacheAttnParams& p, hipStream_t stream) {
    const unsigned tiles = (unsigned)(p.batch * p.c.heads * p.tiles);
    if (!grid_fits(tiles, p.rows_of_tile > 32 ? kCacheTileWaves * 64 : kCacheWaves * 64)) return hipErrorInvalidConfiguration;
    if (p.rows_of_tile == 16) return launch_kernel(&cache_token_kernel<DT, CT, DH>, dim3(tiles, (unsigned)p.slices), dim3(kCacheWaves * 64), stream, p);
    if (p.rows_of_tile == 32) return launch_kernel(&cache_rows_kernel<DT, CT, DH>, dim3(tiles, (unsigned)p.slices), dim3(kCacheWaves * 64), stream, p);
    constexpr int QW = kCacheTileWaves;
    const hipError_t e = launch_kernel(&cache_tile_kernel<DT, CT, DH, QW>, dim3(tiles, (unsigned)p.slices), dim3(QW * 64), stream, p);
    if (e != hipSuccess || p.slices == 1) return e;
    return launch_kernel(&cache_join_kernel<DT, DH, QW>, dim3(tiles, QW), dim3(256), stream, p);
}
hipError_t launch_cache_attention(const CacheAttnParams& p, int dt, int ct, int d, hipStream_t stream) {
#define TIR_CACHE(DT, CT, DH) if (dt == DT && ct == CT && d == DH) return launch_cache_as<DT, CT, DH>(p, stream);
    TIR_CACHE(DT_F16, CT_I8, 64) TIR_CACHE(DT_F16, CT_I8, 128) TIR_CACHE(DT_F16, CT_E4M3, 64) TIR_CACHE(DT_F16, CT_E4M3, 128)
    TIR_CACHE(DT_BF16, CT_I8, 64) TIR_CACHE(DT_BF16, CT_I8, 128) TIR_CACHE(DT_BF16, CT_E4M3, 64) TIR_CACHE(DT_BF16, CT_E4M3, 128)
#undef TIR_CACHE
    return hipErrorInvalidValue;
}

// Tile of rows and number of workgroups that share a tile's keys.  How many keys a sequence holds is known on the device only: the table's columns bound it, and slices that
// a short sequence does not need end at once.
//
// Tiles of 32 rows and of 256, us: 4 x 509 tokens x 32 query heads (8 key heads) of 128 over 4 thousand, e4m3 176 / 148, int8 and bf16 203 / 150, heads of 64 112 / 99; from fewer rows or workgroups the
// small ones are as fast or faster: 1000 tokens over themselves 34.9 / 39.4, 64 x 20 tokens over 2500 139 / 187, 16 x 200 x 16 heads of 64 over 1200 42 / 56.
//
// A table much wider than the sequences lets the 256-row tiles count slices that then have no keys.  130 tokens x 16 query heads (4 key heads) of 128 in a table of 200 000 positions, tiles of 32 and of 256, us:
// holding 130 6.3 / 14.1, 1000 15.0 / 19.1, 4000 25.3 / 26.5, 16 000 56.0 / 46.0, 200 000 541 / 344.  The columns do not tell these apart; what a wide table costs a short prompt is less than what narrow tiles cost a
// long one.  Single tokens gain from it: 1 x 777 x 8 heads of 64 7.1 us in a table of its length, 6.4 in a wide one (one chunk per wave instead of two).
static void choose_cache_kernel(CacheAttnParams* p, int64_t d, const StreamWorkspace& ws) {
    const int64_t heads = (int64_t)p->batch * p->c.heads, rows = (int64_t)p->T * p->G, keys = (int64_t)p->c.cols << p->c.shift;
    const int64_t part = d == 64 ? cache_partial_bytes<64>() : cache_partial_bytes<128>();
    // tiles of 256 rows: one workgroup per CU, of which the tile's slices are to fill nearly all
    const int64_t tall = heads * ((rows + 32 * kCacheTileWaves - 1) / (32 * kCacheTileWaves));
    int64_t tall_slices = 1;
    if (ws.partial && tall < 128) {
        tall_slices = 256 / tall;
        if (tall_slices > keys / 256) tall_slices = keys / 256;
        if (tall_slices > ws.bytes / (tall * kCacheTileWaves * part)) tall_slices = ws.bytes / (tall * kCacheTileWaves * part);
        if (tall_slices < 1) tall_slices = 1;
    }
    int64_t tiles = heads * ((rows + 31) / 32), slices = 1;
    p->rows_of_tile = rows <= 16 ? 16 : 32;
    if (rows >= 512 && tall * tall_slices >= 192) {
        p->rows_of_tile = 32 * kCacheTileWaves;
        tiles = tall;
        slices = tall_slices;
    } else if (ws.partial && tiles <= ws.counters && tiles < 512) {
        // Tiles of 16 rows: as many workgroups as CUs, with two chunks of 64 keys per wave.  256 and 512 workgroups in all, us: one token over 30 000 20.8 / 25.3, over 200 003 87 / 96, 32 x 2000 20.3 / 24.0;
        // one chunk per wave 8 x 2000 15.9, two 14.2.  Tiles of 32: twice the workgroups, two chunks of 32 (8 x 20 tokens over 3000 27.1 us, 33.9 with one workgroup per CU and four).
        const bool token = p->rows_of_tile == 16;
        const int64_t small = !token ? part : d == 64 ? token_partial_bytes<64>() : token_partial_bytes<128>();
        const int64_t room = token ? 256 : 512, least = token ? 512 : 256;
        slices = (room + tiles - 1) / tiles;
        if (slices > (keys + least - 1) / least) slices = (keys + least - 1) / least;
        if (slices > 64) slices = 64;
        if (slices > ws.bytes / (tiles * small)) slices = ws.bytes / (tiles * small);
        if (slices < 1) slices = 1;
    }
    p->tiles = (int)(tiles / heads);
    p->slices = (int)slices;
    if (slices > 1) {
        p->ws = ws.partial;
        p->ws_count = ws.count;
    }
    const FastDiv dt = make_fastdiv((unsigned)p->tiles);
    p->div_tiles_magic = dt.magic; p->div_tiles_shift = dt.shift;
}

static tir_status check_cache(const char* who, const tir_kv_cache* c, int64_t batch, CacheView* out) {
    if (!c) return host_error(TIR_ERR_INVALID_ARG, "%s: cache is null", who);
    if (c->dtype != TIR_I8 && c->dtype != TIR_E4M3) return host_error(TIR_ERR_UNSUPPORTED, "%s: cache dtype %d (I8 and E4M3 are compiled)", who, (int)c->dtype);
    if (c->d != 64 && c->d != 128) return host_error(TIR_ERR_UNSUPPORTED, "%s: head dimension %lld (64 and 128 are compiled)", who, (long long)c->d);
    int shift = 0;
    for (int s = 4; s <= 7; ++s)
        if (c->block_tokens == (1 << s)) shift = s;
    if (!shift) return host_error(TIR_ERR_UNSUPPORTED, "%s: blocks of %lld tokens (16, 32, 64 and 128 are compiled)", who, (long long)c->block_tokens);
    if (c->blocks < 1 || c->heads < 1 || c->columns < 1) return host_error(TIR_ERR_INVALID_ARG, "%s: cache of %lld blocks, %lld heads and %lld columns: at least one of each is needed", who, (long long)c->blocks, (long long)c->heads, (long long)c->columns);
    // (positions a few chunks behind the last one are computed with 31 bits)
    if (c->blocks > kMax31 || c->heads > 65535 || c->columns > ((kMax31 - 65535) >> shift)) return host_error(TIR_ERR_UNSUPPORTED, "%s: blocks beyond 2^31-1, columns * block_tokens beyond 2^31-2^16 or more than 65535 heads", who);
    if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->table) return host_error(TIR_ERR_INVALID_ARG, "%s: a pointer of the cache is null", who);
    if (!host_aligned(c->k, 16) || !host_aligned(c->v, 16)) return host_error(TIR_ERR_ALIGNMENT, "%s: the cache's k and v must be 16-byte aligned", who);
    if (!host_aligned(c->k_scale, 4) || !host_aligned(c->v_scale, 4) || !host_aligned(c->table, 4)) return host_error(TIR_ERR_ALIGNMENT, "%s: the cache's scales and table must be 4-byte aligned", who);
    if (batch > c->sequences) return host_error(TIR_ERR_INVALID_ARG, "%s: batch of %lld, the cache's table has %lld sequences", who, (long long)batch, (long long)c->sequences);
    out->k = (char*)c->k;
    out->v = (char*)c->v;
    out->ks = c->k_scale;
    out->vs = c->v_scale;
    out->table = c->table;
    out->blocks = (int)c->blocks;
    out->heads = (int)c->heads;
    out->cols = (int)c->columns;
    out->shift = shift;
    return TIR_OK;
}

}  // namespace tir

using namespace tir;

extern "C" {

tir_status tir_cache_append(const tir_kv_cache* cache, const void* K, const void* V, const int32_t* start,
                            const int32_t* count, int64_t batch, int64_t T, int64_t k_bs, int64_t k_rs, int64_t k_hs,
                            int64_t v_bs, int64_t v_rs, int64_t v_hs, tir_dtype in, tir_stream stream) {
    const char* const who = "cache append";
    if ((int)in < 0 || (int)in > TIR_E4M3) return host_error(TIR_ERR_INVALID_ARG, "unknown dtype code (in=%d)", (int)in);
    if (in != TIR_F16 && in != TIR_BF16) return host_error(TIR_ERR_UNSUPPORTED, "%s: unsupported input dtype %d", who, (int)in);
    if (batch < 0 || T < 0) return host_error(TIR_ERR_INVALID_ARG, "negative extent (batch=%lld T=%lld)", (long long)batch, (long long)T);
    AppendParams p = {};
    tir_status st = check_cache(who, cache, batch, &p.c);
    if (st == TIR_OK) st = check_row_strides(who, "K", k_bs, k_rs, k_hs);
    if (st == TIR_OK) st = check_row_strides(who, "V", v_bs, v_rs, v_hs);
    if (st != TIR_OK) return st;
    if (batch == 0 || T == 0) return TIR_OK;
    if (!K || !V || !start) return host_error(TIR_ERR_INVALID_ARG, "%s: K, V or start is null", who);
    if (!host_aligned(K, 16) || !host_aligned(V, 16)) return host_error(TIR_ERR_ALIGNMENT, "%s: K and V must be 16-byte aligned", who);
    if (!host_aligned(start, 4) || !host_aligned(count, 4)) return host_error(TIR_ERR_ALIGNMENT, "%s: start and count must be 4-byte aligned", who);
    if (T > kMax31 - 128 || batch > kMax31) return host_error(TIR_ERR_UNSUPPORTED, "extent beyond 2^31-1");
    int64_t touched = (T + (1 << p.c.shift) - 2) / (1 << p.c.shift) + 1;      // T tokens from any position on
    if (touched > p.c.cols) touched = p.c.cols;
    if (batch * touched > kMax31 / p.c.heads) return host_error(TIR_ERR_UNSUPPORTED, "%s: too many blocks in one call", who);
    p.K = K; p.V = V;
    p.k_bs = k_bs; p.k_rs = k_rs; p.k_hs = k_hs;
    p.v_bs = v_bs; p.v_rs = v_rs; p.v_hs = v_hs;
    p.start = start; p.count = count;
    p.T = (int)T;
    p.touched = (int)touched;
    const FastDiv dh = make_fastdiv((unsigned)p.c.heads), dt = make_fastdiv((unsigned)touched);
    p.div_h_magic = dh.magic; p.div_h_shift = dh.shift;
    p.div_t_magic = dt.magic; p.div_t_shift = dt.shift;
    const hipError_t e = launch_append(p, (int)in, cache->dtype == TIR_I8 ? CT_I8 : CT_E4M3, (int)cache->d, batch, (hipStream_t)stream);
    if (e != hipSuccess) return launch_error(who, e);
    return TIR_OK;
}

tir_status tir_cache_attention(const void* Q, const tir_kv_cache* cache, void* O, const int32_t* lens,
                               const int32_t* count, int64_t batch, int64_t T, int64_t Hq, int64_t q_bs, int64_t q_rs,
                               int64_t q_hs, int64_t o_bs, int64_t o_rs, int64_t o_hs, float scale, tir_dtype in,
                               tir_dtype out, tir_stream stream) {
    const char* const who = "cache attention";
    if ((int)in < 0 || (int)in > TIR_E4M3 || (int)out < 0 || (int)out > TIR_E4M3) return host_error(TIR_ERR_INVALID_ARG, "unknown dtype code (in=%d out=%d)", (int)in, (int)out);
    if (!((in == TIR_F16 || in == TIR_BF16) && (out == in || out == TIR_F32))) return host_error(TIR_ERR_UNSUPPORTED, "%s: unsupported (in, out) dtype pair (%d, %d)", who, (int)in, (int)out);
    if (batch < 0 || T < 0 || Hq < 0) return host_error(TIR_ERR_INVALID_ARG, "negative extent (batch=%lld T=%lld Hq=%lld)", (long long)batch, (long long)T, (long long)Hq);
    CacheAttnParams p = {};
    tir_status st = check_cache(who, cache, batch, &p.c);
    if (st == TIR_OK) st = check_row_strides(who, "Q", q_bs, q_rs, q_hs);
    if (st == TIR_OK) st = check_row_strides(who, "O", o_bs, o_rs, o_hs);
    if (st != TIR_OK) return st;
    st = check_scale(who, scale);
    if (st != TIR_OK) return st;
    if (Hq % p.c.heads) return host_error(TIR_ERR_INVALID_ARG, "%s: %d key heads do not divide %lld query heads", who, p.c.heads, (long long)Hq);
    if (batch == 0 || T == 0 || Hq == 0) return TIR_OK;
    if (!Q || !O || !lens) return host_error(TIR_ERR_INVALID_ARG, "%s: Q, O or lens is null", who);
    if (!host_aligned(Q, 16) || !host_aligned(O, 16)) return host_error(TIR_ERR_ALIGNMENT, "%s: Q and O must be 16-byte aligned", who);
    if (!host_aligned(lens, 4) || !host_aligned(count, 4)) return host_error(TIR_ERR_ALIGNMENT, "%s: lens and count must be 4-byte aligned", who);
    if ((batch > 1 && o_bs == 0) || (T > 1 && o_rs == 0) || (Hq > 1 && o_hs == 0)) return host_error(TIR_ERR_INVALID_ARG, "%s: a stride of O is zero: its rows overlap", who);
    if (T > kMax31 || Hq > kMax31 || T > (kMax31 - 512) / (Hq / p.c.heads)) return host_error(TIR_ERR_UNSUPPORTED, "extent beyond 2^31-1");
    p.G = (int)(Hq / p.c.heads);
    p.T = (int)T;
    if (batch > kMax31 / p.c.heads || batch * p.c.heads > kMax31 / ((T * p.G + 31) / 32)) return host_error(TIR_ERR_UNSUPPORTED, "%s: too many tiles of queries", who);
    p.batch = (int)batch;
    p.Q = Q; p.O = O;
    p.q_bs = q_bs; p.q_rs = q_rs; p.q_hs = q_hs;
    p.o_bs = o_bs; p.o_rs = o_rs; p.o_hs = o_hs;
    p.lens = lens; p.count = count;
    p.out32 = out == TIR_F32;
    p.scale_log2e = scale * 1.44269504088896340736f;
    const FastDiv dg = make_fastdiv((unsigned)p.G), dh = make_fastdiv((unsigned)p.c.heads);
    p.div_g_magic = dg.magic; p.div_g_shift = dg.shift;
    p.div_h_magic = dh.magic; p.div_h_shift = dh.shift;
    const StreamWorkspace ws = stream_workspace((hipStream_t)stream);
    choose_cache_kernel(&p, cache->d, ws);
    const hipError_t e = launch_cache_attention(p, (int)in, cache->dtype == TIR_I8 ? CT_I8 : CT_E4M3, (int)cache->d, (hipStream_t)stream);
    if (e != hipSuccess) return launch_error(who, e);
    return TIR_OK;
}

const char* tir_debug_cache_kernel(int64_t batch, int64_t T, int64_t Hq, int64_t heads, int64_t d, int64_t block_tokens, int64_t columns) {
    static thread_local char name[48];
    CacheAttnParams p = {};
    if (batch < 1 || T < 1 || heads < 1 || Hq < heads || columns < 1 || heads > 65535 || Hq > kMax31 || T > (kMax31 - 512) / (Hq / heads) || batch > kMax31 / heads ||
        batch * heads > kMax31 / ((T * (Hq / heads) + 31) / 32) || columns > (kMax31 - 65535) / 128 || (d != 64 && d != 128) || (block_tokens != 16 && block_tokens != 32 && block_tokens != 64 && block_tokens != 128)) return "";
    p.batch = (int)batch;
    p.T = (int)T;
    p.G = (int)(Hq / heads);
    p.c.heads = (int)heads;
    p.c.cols = (int)columns;
    while ((16ll << p.c.shift) < block_tokens * 16) ++p.c.shift;
    // (a registered workspace, as the variant queries of the products assume one)
    const StreamWorkspace ws = {(void*)256, nullptr, (int64_t)(tir_workspace_bytes() / (1 << 20)) << 20, 16384};
    choose_cache_kernel(&p, d, ws);
    snprintf(name, sizeof name, "rows%d/z%d", p.rows_of_tile, p.slices);
    return name;
}

}  // extern "C"
