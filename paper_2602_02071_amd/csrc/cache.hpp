// The paged 8-bit key/value cache: its layout and the launch descriptors of
// its operators.
//
// K and V are FP8 E4M3 codes in pages of `page` tokens (16, 32, 64 or 128).
// Every (page, key/value head) has one power-of-two scale for K and one for V,
// kept as the biased exponent byte e: the value is code * 2^(e - 127), exact in
// bf16 for every finite code (4 significant bits, |exponent| < 127), so a
// conversion with its scale costs one instruction per two elements and rounds
// nothing.  K keeps rows of D bytes per token; V keeps groups of 16 tokens
// transposed, [D][16]: the operand of P V takes 8 or 16 consecutive keys of
// one d, which this order gives to one 16-byte load.
#pragma once
#include "common.hpp"

namespace baps {

// bounds of the scale exponents: with them every dequantised value is a
// normal bf16 number (2^-9 * 2^-100 up to 448 * 2^119)
constexpr int kCacheExpLo = 27, kCacheExpHi = 246;

struct CacheView {                  // one layer of the pool
    uint8_t *k, *v;                 // [num_pages][Hkv][page][D], [num_pages][Hkv][page/16][D][16]
    uint8_t *ke, *ve;               // [num_pages][Hkv]
    int num_pages, Hkv, lpage;      // lpage: log2(page)
};

struct CacheAppendParams {
    CacheView c;
    const uint16_t *k, *v;          // new tokens, bf16: token t, head h, element d at t*stride + h*D + d
    long long stride;
    const int *cu, *lens, *table;
    int table_width, B, max_new, total;
};

struct CacheAttnParams {
    CacheView c;
    const uint16_t* q;              // row t, head h, element d at t*qstride + h*D + d
    long long qstride;
    uint16_t* o;                    // [total_q][Hq][D] bf16
    float* lse;                     // [total_q][Hq] or null
    const int *cu, *lens, *table;
    int table_width, B, Hq, total_q, max_q, max_len;
    int window, sinks;              // window 0: none
    float scale;                    // score scale in log2 units
    bool once;                      // the cache is read once and does not stay in the caches on the way
    int chunk;                      // > 0: places of sequence_of_place (cache_attention.hip)
    int nsplit;                     // > 1: partial results go to part / ml
    float* part;                    // [nsplit][total_q * Hq][D] unnormalised sums
    float* ml;                      // [nsplit][total_q * Hq][2] running maximum (log2 units) and sum
};

struct CacheForkParams {
    uint8_t *k, *v, *ke, *ve;       // the whole pool
    int layers, num_pages, Hkv, page, D;
    const int* table_in;            // [B_in][width]
    const int* lens_in;
    const int* refs_in;
    const int *parent, *grow;       // [B_out]; grow may be null
    int *table_out, *lens_out, *refs_out, *missing;
    int B_in, B_out, width;
    int *src, *dst, *taken, *over, *fresh;  // workspace, [B_out] each; fresh: [B_out + 1]
};

struct CacheCompactParams {
    uint8_t *k, *v, *ke, *ve;
    int layers, num_pages, Hkv, page, D;
    const int* refs_in;
    const int* table_in;
    int *refs_out, *table_out, *remap, *live;
    long long entries;              // table entries (rows * width)
    int *from, *to, *held;          // workspace, [num_pages] each
    int* moves;                     // workspace: how many pages move
};

hipError_t launch_cache_append(const CacheAppendParams& p, int D, hipStream_t st);
hipError_t launch_cache_attention(const CacheAttnParams& p, int D, hipStream_t st);
hipError_t launch_cache_fork(const CacheForkParams& p, hipStream_t st);
hipError_t launch_cache_compact(const CacheCompactParams& p, hipStream_t st);

// The split of the attention call: how many key splits, for how many keys at
// most that a row reaches
int cache_attention_splits(int B, int Hq, int Hkv, int D, int total_q, int max_q, int max_len, int window, int sinks,
                           int ncu);

}  // namespace baps
