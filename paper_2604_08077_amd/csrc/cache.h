// The paged key/value cache: its geometry on the device side, and the launchers of its kernels (cache.hip, decode.hip).
//
// Layout: K and V each [pages][kv_heads][page_size][head_dim], so that a page's tokens of one head lie one behind the other (a
// decode step of one head reads runs of page_size rows); in 8 bits (e4m3) a scale per token and head, fp32
// [pages][kv_heads][page_size].  Position p of sequence s lies in page table[s][p / page_size].  A table entry that is no
// page of the cache, and positions beyond a table row, hold no token: not written, read as zero, attended by nobody.
#pragma once
#include "geom.h"

namespace adaspark {

constexpr int CACHE_THREADS = 256;  // of a workgroup of the write and read kernels

struct CacheGeom {
    int B, pages, shift, table_pages;  // page_size = 1 << shift
    int Hq, Hkv, G, D;
    bool e4m3;
};

inline CacheGeom make_cache_geom(const adaspark_cache &c)
{
    CacheGeom g;
    g.B = c.sequences;
    g.pages = c.pages;
    g.shift = __builtin_ctz((unsigned)c.page_size);
    g.table_pages = c.table_pages;
    g.Hq = c.q_heads;
    g.Hkv = c.kv_heads;
    g.G = c.q_heads / c.kv_heads;
    g.D = c.head_dim;
    g.e4m3 = c.format == ADASPARK_CACHE_E4M3;
    return g;
}

struct CacheData {
    void *K, *V;
    float *ks, *vs;  // null in bf16
};

hipError_t launch_cache_write(const CacheGeom &g, int tokens, const uint16_t *K, long long k_stride, const uint16_t *V,
                              long long v_stride, const int32_t *starts, const int32_t *table, const int32_t *lengths,
                              const CacheData &c, hipStream_t st);
hipError_t launch_cache_read(const CacheGeom &g, int tokens, const int32_t *starts, const int32_t *table, const CacheData &c,
                             uint16_t *K, uint16_t *V, hipStream_t st);
size_t decode_workspace_bytes(const CacheGeom &g);
hipError_t launch_decode_attn(const CacheGeom &g, const uint16_t *Q, const int32_t *table, const int32_t *lengths,
                              const CacheData &c, uint16_t *O, float *lse, void *ws, hipStream_t st);

}  // namespace adaspark
