// The 8-bit paged K/V cache as the kernels see it: its arrays, the layout of a page, and what its entry points check alike.
#pragma once

#include "hgf_common.cuh"

namespace hgf {

constexpr int kCacheBlock = HGF_CACHE_BLOCK;              // tokens of a page
constexpr unsigned int kStatusCache = 0x40000000u;        // status word: a cache call met an index outside its arrays
constexpr int kCacheMaxSeqs = HGF_CACHE_MAX_SEQS;

// A page holds, for each head, 3 * 64 * DH bytes: the codes of K1 and K2, [64 tokens][DH] each, and of V transposed, [DH][64 tokens].  Each of
// the three is cut into tiles of 16 rows by 32 columns, 512 bytes, the column tiles of a row tile side by side.  A tile is stored as the 32 lanes
// of a warp take it as the left operand of an m16n8k32 product: with row 8 a + g and column 16 h + 4 t + b, byte (4 g + t) * 16 + 8 h + 4 a + b, so
// a lane's sixteen bytes are one 128-bit load and a product over 32 dims (scores) or 32 tokens (values) needs no byte moved.
__host__ __device__ inline int cache_tile_byte(int row, int col, int cols) {
    return (((row >> 4) * (cols >> 5) + (col >> 5)) * 32 + (row & 7) * 4 + ((col >> 2) & 3)) * 16 + ((col >> 4) & 1) * 8 + ((row >> 3) & 1) * 4 + (col & 3);
}
// Rows of the open block ([64][DH] bf16): the eights of row r are stored at place (their index) ^ (r & 7), which spreads eight rows' loads of one
// eight over all shared-memory banks.
__host__ __device__ inline int cache_open_eight(int row, int eight) { return eight ^ (row & 7); }

struct CacheView {
    int8_t *codes;           // [n_pages][H][3 * 64 * DH]
    float4 *scales;          // [n_pages][H]: K1, K2, V, 0
    __nv_bfloat16 *open;     // [n_slots][H][3][64][DH]
    int32_t *table;          // [n_slots][max_pages]
    int32_t *held, *length;  // [n_slots]
    int32_t *refs;           // [n_pages]
    int32_t *arrivals;       // [n_slots], zero between calls
    int n_pages, n_slots, max_pages, H;
};

// Checks a cache's description and the list length of a call on it.
hgf_status parse_cache(const hgf_cache *c, int64_t n, CacheView *v);

// What a slot holds is used only if it is consistent: pages assigned within the table, a length that these pages and the open block can hold.
__device__ __forceinline__ bool cache_slot_ok(const CacheView &c, int held, int length) {
    return held >= 0 && held <= c.max_pages && length >= 0 && (length >> 6) <= held;
}

// Whether entry i of a list of slots is the first that names its slot.
__device__ __forceinline__ bool cache_first_of(const int32_t *__restrict__ slots, int i, int slot) {
    bool again = false;
    for (int j = threadIdx.x; j < i; j += blockDim.x) again = again || slots[j] == slot;
    return !__syncthreads_or(again);
}

}  // namespace hgf
