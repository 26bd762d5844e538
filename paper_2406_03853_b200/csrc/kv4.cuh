// Where things are in the 4-bit key / value cache (eesd_kv4).
#pragma once
#include "../../include/eesd.h"
#include "common.cuh"

namespace eesd {
namespace kv4 {

struct Cache {
    unsigned char *pool;
    const int32_t *table;
    int64_t table_stride;
    int n_pages, max_pages, Hkv;
    int shift;   // log2 of a page's tiles
};

// bytes of a tile of 16 tokens and where its parts begin
template <int D, int G> struct Tile {
    static constexpr int V = 8 * D, SCALES = 16 * D, KZ = SCALES + 64 * G, VZ = KZ + 16 * G, BYTES = VZ + 16 * G;
};

// tile `tile` (>= 0) of head h of sequence b; NULL where its page does not exist
__device__ __forceinline__ unsigned char *tile_at(const Cache &c, int b, int h, int64_t tile, int tile_bytes) {
    const int64_t p = tile >> c.shift;
    if (p >= c.max_pages) return nullptr;
    const int page = c.table[b * c.table_stride + p];
    if ((unsigned)page >= (unsigned)c.n_pages) return nullptr;
    return c.pool + ((((size_t)page * c.Hkv + h) << c.shift) + (size_t)(tile & ((1 << c.shift) - 1))) * tile_bytes;
}

// (x, y) turned by (cos, sin): each operation rounded by itself
__device__ __forceinline__ float2 turn(float x, float y, float2 cs) {
    return make_float2(__fsub_rn(__fmul_rn(x, cs.x), __fmul_rn(y, cs.y)), __fadd_rn(__fmul_rn(x, cs.y), __fmul_rn(y, cs.x)));
}

}  // namespace kv4

int kv4_open(const eesd_kv4 *c, const void *pool, size_t pool_bytes, const eesd_kv4_rows *r, kv4::Cache *out, eesd_kv4_layout *l);
int kv4_rows_check(const eesd_kv4_tensor *t, int dtype);
}  // namespace eesd
