// Attention over the paged 8-bit cache, eq. (2) in fp32 (the "Default" setup):
//   S = q.k / sqrt(D), P = 2^(S log2 e - m), O = sum P v / sum P,
// with the online maximum m, over the keys that a row sees: those up to its
// own position, of them the last `window` and the first `sinks`.
//
// The dequantised values code * 2^(e-127) are exact in bf16 (cache.hpp), so
// both products run on bf16 MFMA with fp32 sums and the only roundings are P's
// and the output's.
//
// Two kernels.  rows: up to 16 flattened (query position, head of the group)
// rows of a key/value head per workgroup, for decode; bound by the cache's
// bytes.  tile: 128 or 256 rows per workgroup, for chunks of a prompt; bound by the
// matrix unit and the exponentials.  Either splits the keys of a row over
// workgroups where rows alone are too few, and combine joins the parts.
#include <algorithm>
#include <type_traits>

#include "cache.hpp"
#include "combine.hpp"
#include "tile_core.hpp"

namespace baps {

namespace {

typedef __bf16 bf16x2e __attribute__((ext_vector_type(2)));

// eight codes (two words) times 2^(e-127), e given as that power's fp32 value
__device__ __forceinline__ u32x4 dequant8(uint32_t a, uint32_t b, float s)
{
    return u32x4{__builtin_bit_cast(uint32_t, (bf16x2e)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, false)),
                 __builtin_bit_cast(uint32_t, (bf16x2e)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, true)),
                 __builtin_bit_cast(uint32_t, (bf16x2e)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, false)),
                 __builtin_bit_cast(uint32_t, (bf16x2e)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, true))};
}

__device__ __forceinline__ float pow2_of_byte(int e) { return hif8::u2f((uint32_t)e << 23); }

// the larger of the values of lanes l and l ^ 16
__device__ __forceinline__ float max_quarters(float x)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return fmaxf(hif8::u2f(r[0]), hif8::u2f(r[1]));
}

// A sequence's new tokens and length, held to what the buffers have.
struct Seq {
    int c0, n, first, len;          // packed rows [c0, c0 + n) at positions first ..; keys [0, len)
};

__device__ __forceinline__ Seq sequence(const CacheAttnParams& p, int b)
{
    Seq s;
    const int c1 = p.cu[b + 1], len = min(max(p.lens[b], 0), 1 << 30);
    s.c0 = p.cu[b];
    s.n = s.c0 < 0 || c1 <= s.c0 || c1 > p.total_q ? 0 : c1 - s.c0;
    s.first = len - s.n;
    s.n = min(s.n, p.max_q);
    s.len = (int)min((long long)len, (long long)p.table_width << p.c.lpage);
    return s;
}

// Of the 16 keys from k0 on, those up to t_hi that are in the window of the
// lowest row (lo) or sinks, as bits; none where the group has no page.
__device__ __forceinline__ uint32_t keys_seen(int k0, int t_hi, int lo, int sinks, bool bad)
{
    auto below = [&](int x) { return (1u << min(max(x - k0, 0), 16)) - 1u; };
    return bad ? 0u : below(t_hi + 1) & (~below(lo) | below(sinks));
}

// Byte mask of word w of a 16-key group
__device__ __forceinline__ uint32_t byte_mask(uint32_t seen, int w)
{
    return ((((seen >> (4 * w)) & 15u) * 0x204081u) & 0x01010101u) * 0xffu;
}

// ---------------------------------------------------------------- rows kernel
// A wave takes steps of 64 keys.  S^T = K Q^T on 16x16x32: row r of the 16-key
// tile t is key 16 (r/4) + 4 t + r%4 of the step, so that a lane's 16 scores
// (4 tiles x 4 registers) are the 16 consecutive keys of its lane group: then
// one 16-byte load of V's transposed groups is the lane's operand of
// O^T += V^T P^T, and P never leaves its lane.  K's rows are read as 16 bytes
// per lane, d = 64 j + 16 (lane/16) .., and Q in the same order.  No LDS on
// the way: the loads of step j+1 go out as soon as the registers of step j are
// read.  P enters P V as two bf16 terms (P = hi + lo to 2^-17): the second
// product is free where the bytes bound the kernel (64 sequences of 5000 to 8192
// keys, GQA 32/8, D = 128: 140 us, 6.2 TB/s).
constexpr int kStep = 64;
constexpr int kRows = 16;
constexpr int kWaves = 4;

// The sequence of place z in the order longest first, every other `chunk` places in
// reverse: the workgroups of one chunk take a CU each, so that a CU's two hold a long
// and a short sequence, and none is done long before the others (64 sequences, GQA
// 32/8, D = 128, of 5000 to 8192 keys: 150 -> 140 us; of 1000 to 9000: 142 -> 111; of
// one length: 136 -> 139).  One lane per sequence; B <= 64.
__device__ __forceinline__ int sequence_of_place(const CacheAttnParams& p, int z, int chunk, int lane)
{
    // (different for all, so that every place has one)
    const uint32_t key = lane < p.B ? (uint32_t)min(max(p.lens[lane], 0), (1 << 26) - 1) << 6 | (63 - lane) : 0;
    int rank = 0;
#pragma unroll 4
    for (int j = 0; j < p.B; ++j) rank += (uint32_t)__builtin_amdgcn_readlane(key, j) > key ? 1 : 0;
    const int first = z / chunk * chunk, last = min(first + chunk, p.B) - 1;
    const int want = (z / chunk) & 1 ? first + last - z : z;
    return __builtin_ctzll(__ballot(lane < p.B && rank == want));
}

template <int D, int TR, bool ONCE>
__global__ __launch_bounds__(64 * kWaves, 2) void baps_cache_rows_kernel(CacheAttnParams p)
{
    constexpr int kJ = D / 64;                                  // 16-byte pieces of a K row per lane
    constexpr int kDT = D / 16;                                 // 16-wide d tiles of O^T
    constexpr int kTile = kRows * TR;
    __shared__ float ldo[kWaves - 1][kTile][D];
    __shared__ float ldm[kWaves][kTile], ldl[kWaves][kTile];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, grp = lane >> 4;
    const int G = p.Hq / p.c.Hkv;
    const int split = blockIdx.x;
    const int h = blockIdx.y % p.c.Hkv, tile = blockIdx.y / p.c.Hkv;
    int b = blockIdx.z;
    if (p.chunk > 0) b = sequence_of_place(p, b, p.chunk, lane);
    const Seq s = sequence(p, b);
    const int f0 = tile * kTile, flat = s.n * G;
    if (f0 >= flat) return;

    // positions of the workgroup's rows (a window counts from them, also behind the
    // table's end) and the last key
    const int t_lo = s.first + f0 / G, p_hi = s.first + min(flat - 1, f0 + kTile - 1) / G, t_hi = min(p_hi, s.len - 1);
    // the lane's rows: c16 of each of the TR row tiles
    bool row_ok[TR];
    int pos[TR];
    long long row[TR];
    u32x4 qop[TR][2 * kJ];
#pragma unroll
    for (int x = 0; x < TR; ++x) {
        row_ok[x] = f0 + kRows * x + c16 < flat;
        const int f = row_ok[x] ? f0 + kRows * x + c16 : f0;
        const int i = f / G, hq = h * G + f % G;
        pos[x] = row_ok[x] ? s.first + i : -1;
        row[x] = (long long)(s.c0 + i) * p.Hq + hq;
#pragma unroll
        for (int k = 0; k < 2 * kJ; ++k)
            qop[x][k] = *reinterpret_cast<const u32x4*>(p.q + (s.c0 + i) * p.qstride + hq * D + 64 * (k >> 1) + 16 * grp + 8 * (k & 1));
    }

    const KeyBlocks kb = key_blocks<kStep>(t_lo, t_hi, p.window, p.sinks);
    const int per = (kb.n + p.nsplit - 1) / p.nsplit;
    const int j1 = min(kb.n, (split + 1) * per);
    int j = split * per + wave;

    const int* trow = p.table + (long long)b * p.table_width;
    const int lp = p.c.lpage, page_mask = (1 << lp) - 1;
    const uint32_t page_bytes = (uint32_t)D << lp;
    const float ninf = -__builtin_huge_valf();
    float m[TR], l[TR];
    f32x4 oacc[TR][kDT];
#pragma unroll
    for (int x = 0; x < TR; ++x) {
        m[x] = ninf;
        l[x] = 0.0f;
#pragma unroll
        for (int t = 0; t < kDT; ++t) oacc[x][t] = f32x4{};
    }

    // The lane's 16-token group of a step is c16 / 4 in K and grp in V; what
    // depends on the lane is a constant offset into the page.  The page is looked
    // up one step ahead of its codes, so that no load waits for the table.
    const int kslot = 16 * (c16 >> 2) >> lp, vslot = 16 * grp >> lp;
    const uint32_t kin = ((16 * (c16 >> 2) & page_mask) + (c16 & 3)) * D + 16 * grp;
    const uint32_t vin = (16 * grp & page_mask) * D + 16 * c16;
    struct Codes {                                              // a step's K or V, and its scale
        u32x4 w[kDT];                                           // K: [tile t][piece k] at t * kJ + k
        uint32_t e;
        bool bad;
    };
    static_assert(4 * kJ == kDT, "K and V of a step take the same registers");
    int kpage = 0, vpage = 0;
    auto look = [&](int jj, int slot) { return trow[(uint32_t)min((kb.block(jj) * kStep >> lp) + slot, p.table_width - 1)]; };
    // (a page that is none is read as the last one, and masked)
    auto page_head = [&](int page) { return min((uint32_t)page, (uint32_t)p.c.num_pages - 1u) * (uint32_t)p.c.Hkv + (uint32_t)h; };
    auto load16 = [](const uint8_t* at) {
        const u32x4* q = reinterpret_cast<const u32x4*>(at);
        return ONCE ? __builtin_nontemporal_load(q) : *q;
    };
    auto load_k = [&](Codes& c, int jj) {
        const uint32_t ph = page_head(kpage);
        const uint8_t* at = p.c.k + (kb.block(jj) * kStep & page_mask) * D + ((uint64_t)ph * page_bytes + kin);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int k = 0; k < kJ; ++k) c.w[t * kJ + k] = load16(at + 4 * t * D + 64 * k);
        c.e = p.c.ke[ph];
    };
    auto load_v = [&](Codes& c, int jj) {
        const uint32_t ph = page_head(vpage);
        const uint8_t* at = p.c.v + (kb.block(jj) * kStep & page_mask) * D + ((uint64_t)ph * page_bytes + vin);
#pragma unroll
        for (int t = 0; t < kDT; ++t) c.w[t] = load16(at + 256 * t);
        c.e = p.c.ve[ph];
        c.bad = (unsigned)vpage >= (unsigned)p.c.num_pages;
    };
    // One step: the next step's K is loaded when K's registers are read and V when
    // V's are; at D = 64 with one row tile both ahead of this step, into a second
    // set of registers (64 sequences of 8192 keys: 84 -> 81 us; at D = 128 the
    // second set is one too many, 154 -> 181 us).
    constexpr bool kTwo = TR == 1 && D == 64;
    auto step = [&](Codes& kc, Codes& vc, Codes& kn, Codes& vn) {
        const int key0 = kb.block(j) * kStep;
        const bool more = j + kWaves < j1, more2 = j + 2 * kWaves < j1, bad = vc.bad;
        auto next_k = [&]() {
            load_k(kTwo ? kn : kc, j + kWaves);
            if (more2) kpage = look(j + 2 * kWaves, kslot);
        };
        auto next_v = [&]() {
            load_v(kTwo ? vn : vc, j + kWaves);
            if (more2) vpage = look(j + 2 * kWaves, vslot);
        };
        if (kTwo && more) {
            next_k();
            next_v();
        }
        const float ks = pow2_of_byte(kc.e);
        f32x4 sacc[TR][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int x = 0; x < TR; ++x) sacc[x][t] = f32x4{};
#pragma unroll
            for (int k = 0; k < kJ; ++k) {
                const bf16x8 a = as_bf16x8(dequant8(kc.w[t * kJ + k][0], kc.w[t * kJ + k][1], ks)),
                             b8 = as_bf16x8(dequant8(kc.w[t * kJ + k][2], kc.w[t * kJ + k][3], ks));
#pragma unroll
                for (int x = 0; x < TR; ++x) {
                    sacc[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, as_bf16x8(qop[x][2 * k]), sacc[x][t], 0, 0, 0);
                    sacc[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b8, as_bf16x8(qop[x][2 * k + 1]), sacc[x][t], 0, 0, 0);
                }
            }
        }
        if (!kTwo && more) next_k();
        // Steps that some row does not see whole: scores of hidden keys are
        // -inf, whatever their codes are, and V's codes of keys that no row
        // of the tile sees are zero (what lies behind the last token or in
        // front of the window may be anything, 0 * NaN included).
        if (key0 + kStep - 1 > min(t_lo, t_hi) || (p.window > 0 && key0 <= p_hi - p.window && key0 + kStep > p.sinks) ||
            __any(bad)) {
            // (bitwise conditions: selects and no branches per score)
            const int k0 = key0 + 16 * grp;
            const int snk = p.sinks - k0;
#pragma unroll
            for (int x = 0; x < TR; ++x) {
                const int hi = bad ? -1 : min(pos[x], s.len - 1) - k0, lo = p.window > 0 ? pos[x] - p.window + 1 - k0 : -k0;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int k = 4 * t + r;
                        sacc[x][t][r] = (k <= hi) & ((k >= lo) | (k < snk)) ? sacc[x][t][r] : ninf;
                    }
            }
            const uint32_t seen = keys_seen(k0, t_hi, kb.lo, p.sinks, bad);
#pragma unroll
            for (int t = 0; t < kDT; ++t)
#pragma unroll
                for (int w = 0; w < 4; ++w) vc.w[t][w] &= byte_mask(seen, w);
        }
        u32x4 hi[TR][2], lo[TR][2];
#pragma unroll
        for (int x = 0; x < TR; ++x) {
            float mx = ninf;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sacc[x][t][r]);
            mx = max_halves(max_quarters(mx));
            const float m_new = fmaxf(m[x], mx * p.scale);
            const float nref = m_new == ninf ? 0.0f : -m_new;
            const float fac = m[x] == ninf ? 1.0f : __builtin_amdgcn_exp2f(m[x] - m_new);
            if (__any(fac != 1.0f)) {
#pragma unroll
                for (int t = 0; t < kDT; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) oacc[x][t][r] *= fac;
            }
            l[x] *= fac;
            m[x] = m_new;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                float pr[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    pr[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[x][t][r], p.scale, nref));
                    l[x] += pr[r];
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t w = pack_bf16(pr[2 * e], pr[2 * e + 1]);
                    hi[x][t >> 1][2 * (t & 1) + e] = w;
                    lo[x][t >> 1][2 * (t & 1) + e] = pack_bf16(pr[2 * e] - hif8::u2f(w << 16), pr[2 * e + 1] - hif8::u2f(w & 0xffff0000u));
                }
            }
        }
        const float vs = pow2_of_byte(vc.e);
#pragma unroll
        for (int t = 0; t < kDT; ++t) {
            const bf16x8 v0 = as_bf16x8(dequant8(vc.w[t][0], vc.w[t][1], vs)),
                         v1 = as_bf16x8(dequant8(vc.w[t][2], vc.w[t][3], vs));
#pragma unroll
            for (int x = 0; x < TR; ++x) {
                oacc[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, as_bf16x8(hi[x][0]), oacc[x][t], 0, 0, 0);
                oacc[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, as_bf16x8(hi[x][1]), oacc[x][t], 0, 0, 0);
                oacc[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, as_bf16x8(lo[x][0]), oacc[x][t], 0, 0, 0);
                oacc[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, as_bf16x8(lo[x][1]), oacc[x][t], 0, 0, 0);
            }
        }
        if (!kTwo && more) next_v();
        j += kWaves;
    };
    if (j < j1) {
        Codes ka, va, kb2, vb2;
        kpage = look(j, kslot);
        vpage = look(j, vslot);
        load_k(ka, j);
        load_v(va, j);
        if (j + kWaves < j1) {
            kpage = look(j + kWaves, kslot);
            vpage = look(j + kWaves, vslot);
        }
        while (true) {
            step(ka, va, kb2, vb2);
            if (j >= j1) break;
            if constexpr (kTwo) {
                step(kb2, vb2, ka, va);
                if (j >= j1) break;
            }
        }
    }
    // the waves' parts: a common maximum, then one sum in a fixed order
    float mt[TR];
#pragma unroll
    for (int x = 0; x < TR; ++x) {
        l[x] += __shfl_xor(l[x], 16, 64);
        l[x] += __shfl_xor(l[x], 32, 64);
        if (grp == 0) ldm[wave][kRows * x + c16] = m[x];
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < TR; ++x) {
        const int r16 = kRows * x + c16;
        mt[x] = ldm[0][r16];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) mt[x] = fmaxf(mt[x], ldm[w][r16]);
        const float fac = m[x] == ninf ? 0.0f : __builtin_amdgcn_exp2f(m[x] - mt[x]);
#pragma unroll
        for (int t = 0; t < kDT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) oacc[x][t][r] *= fac;
        l[x] *= fac;
        if (grp == 0) ldl[wave][r16] = l[x];
        if (wave > 0) {
#pragma unroll
            for (int t = 0; t < kDT; ++t) *reinterpret_cast<f32x4*>(&ldo[wave - 1][r16][16 * t + 4 * grp]) = oacc[x][t];
        }
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int x = 0; x < TR; ++x) {
        if (!row_ok[x]) continue;
        const int r16 = kRows * x + c16;
#pragma unroll
        for (int w = 1; w < kWaves; ++w) {
#pragma unroll
            for (int t = 0; t < kDT; ++t) {
                const f32x4 y = *reinterpret_cast<const f32x4*>(&ldo[w - 1][r16][16 * t + 4 * grp]);
#pragma unroll
                for (int r = 0; r < 4; ++r) oacc[x][t][r] += y[r];
            }
            l[x] += ldl[w][r16];
        }
        if (p.nsplit > 1) {
            const long long at = (long long)split * p.total_q * p.Hq + row[x];
#pragma unroll
            for (int t = 0; t < kDT; ++t) *reinterpret_cast<f32x4*>(p.part + at * D + 16 * t + 4 * grp) = oacc[x][t];
            if (grp == 0) {
                p.ml[2 * at] = mt[x];
                p.ml[2 * at + 1] = l[x];
            }
            continue;
        }
        const bool empty = mt[x] == ninf;
        const float inv = empty ? 0.0f : 1.0f / l[x];
#pragma unroll
        for (int t = 0; t < kDT; ++t)
            *reinterpret_cast<u32x2*>(p.o + row[x] * D + 16 * t + 4 * grp) =
                u32x2{pack_bf16(oacc[x][t][0] * inv, oacc[x][t][1] * inv), pack_bf16(oacc[x][t][2] * inv, oacc[x][t][3] * inv)};
        if (p.lse && grp == 0) p.lse[row[x]] = empty ? ninf : 0.69314718055994531f * (mt[x] + log2f(l[x]));
    }
}

// ---------------------------------------------------------------- tile kernel
// NW waves of 32 rows each on the inner loop of tile_core.hpp.  The codes of a
// block come through registers (one 16-byte load of K and of V per thread at D =
// 128), are dequantised once for all waves and stored to LDS as bf16; staging has
// no address arithmetic beyond one 64-bit product, for it is a fifth of a wave's
// instructions.  2048 rows on 32768 keys (GQA 32/8, D = 128): 1207 us in straight
// order, 1157 interleaved, 1051 with the short staging, 1000 with the wave's
// priority raised over the products (1.07 PFLOP/s; without staging it would be
// 908, without the waits for one another 830).

// sum over the wave's lanes (DPP: no LDS round trips)
__device__ __forceinline__ int wave_sum_uniform(int v)
{
#define BAPS_STEP(CTRL, ROWS) v += __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false)
    BAPS_STEP(0x111, 0xF);                                      // row_shr 1, 2, 4, 8: sums up to each lane of 16
    BAPS_STEP(0x112, 0xF);
    BAPS_STEP(0x114, 0xF);
    BAPS_STEP(0x118, 0xF);
    BAPS_STEP(0x142, 0xA);                                      // lane 15 of rows 0 and 2 to rows 1 and 3
    BAPS_STEP(0x143, 0xC);                                      // lane 31 to rows 2 and 3
#undef BAPS_STEP
    return __builtin_amdgcn_readlane(v, 63);
}

// The tiles of all sequences, those that reach furthest first (their keys are
// the work, and the last ones to start set when the call ends): tile `back` of
// sequence b counts from its last one and reaches key lens[b] - back * R / G.
// The place of a workgroup in that order is searched for: tiles that reach x or
// further are counted per sequence without listing any.  Three sequences of
// 2500 to 9001 keys, 777 to 2048 new: 617 -> 547 us against the sequences
// in turn.
struct TileAt {
    int b, back;                    // b < 0: no such tile
};

template <int R>
__device__ __forceinline__ TileAt tile_of_rank(const CacheAttnParams& p, int rank, int G, int lane)
{
    auto tiles = [&](int b) { return (int)(((long long)sequence(p, b).n * G + R - 1) / R); };
    if (p.B == 1) return rank < tiles(0) ? TileAt{0, rank} : TileAt{-1, 0};
    // lane holds sequences lane, lane + 64, ..; the first one's numbers stay in
    // registers
    auto len_of = [&](int b) { return min(max(p.lens[b], 0), 1 << 30); };
    const int len0 = lane < p.B ? len_of(lane) : 0, tiles0 = lane < p.B ? tiles(lane) : 0;
    // tiles of a sequence that reach x
    auto reach_of = [&](int len, int n, int x) {
        const int d = len - x;                                  // (no more than 2^30 apart from zero)
        return d < 0 ? 0 : (int)min((long long)n, ((d + 1LL) * G - 1) / R + 1);
    };
    auto reach = [&](int b, int x) { return b < 64 ? reach_of(len0, tiles0, x) : reach_of(len_of(b), tiles(b), x); };
    auto count = [&](int x) {
        int n = reach_of(len0, tiles0, x);
        for (int b = lane + 64; b < p.B; b += 64) n += reach(b, x);
        return wave_sum_uniform(n);
    };
    // the largest x with more than rank tiles that reach it
    int lo = -p.max_q - 1, hi = len0 + 1;               // (no tile reaches further back than its rows)
    for (int b = lane + 64; b < p.B; b += 64) hi = max(hi, len_of(b) + 1);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) hi = max(hi, __shfl_xor(hi, o, 64));
    hi = __builtin_amdgcn_readfirstlane(hi);
    if (count(lo) <= rank) return TileAt{-1, 0};
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (count(mid) > rank) lo = mid; else hi = mid;
    }
    // among the tiles that reach lo and no further, in the order of the sequences
    int skip = rank - count(lo + 1);
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int b = b0 + lane;
        const int before = b < p.B ? reach(b, lo + 1) : 0;
        const int n = b < p.B ? reach(b, lo) - before : 0;
        int sum = n;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(sum, o, 64);
            if (lane >= o) sum += y;
        }
        const int total = __builtin_amdgcn_readfirstlane(__shfl(sum, 63, 64));
        if (skip < total) {
            const unsigned long long m = __ballot(sum > skip);
            const int l = __builtin_ctzll(m);
            const int back = before + skip - (sum - n);
            return TileAt{b0 + l, __builtin_amdgcn_readfirstlane(__shfl(back, l, 64))};
        }
        skip -= total;
    }
    return TileAt{-1, 0};
}

template <int D, int NW>
__global__ __launch_bounds__(64 * NW, 2) void baps_cache_tile_kernel(CacheAttnParams p)
{
    using Core = TileCore<D, false>;
    constexpr int kTileRows = 32 * NW, kHalf = Core::kHalf, kVBase = Core::kVBase;
    constexpr int kChunks = kBlk * D / 16;                      // 16-byte pieces of codes (512 or 256)
    constexpr int kPer = (kChunks + 64 * NW - 1) / (64 * NW);   // of a thread
    extern __shared__ __attribute__((aligned(1024))) char lds[];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j32 = lane & 31, half = lane >> 5;
    const int G = p.Hq / p.c.Hkv;
    // head fastest: with 8 of them each XCD (workgroups go round-robin over the
    // eight) keeps one head's codes in its L2
    const int h = blockIdx.x % p.c.Hkv;
    const int split = blockIdx.x / p.c.Hkv % p.nsplit;
    const int rank = blockIdx.x / (p.c.Hkv * p.nsplit);
    const TileAt at = tile_of_rank<kTileRows>(p, rank, G, lane);
    if (at.b < 0) return;
    const int b = at.b;
    const Seq s = sequence(p, b);
    const int flat = s.n * G;
    const int tile = (flat + kTileRows - 1) / kTileRows - 1 - at.back;
    if (tile < 0) return;                                       // (the caller's arrays changed meanwhile)
    const int f0 = tile * kTileRows;

    // lanes behind the last row compute it again, and store nothing: no mask for
    // them in the loop (500 tokens on 3800 keys, D = 64: 64 -> 47 us)
    const int wf0 = min(f0 + wave * 32, flat - 1);
    const bool row_ok = f0 + wave * 32 + j32 < flat;
    const int f = min(f0 + wave * 32 + j32, flat - 1), i = f / G, hq = h * G + f % G;
    const int pos = min(s.first + i, s.len - 1);
    const int win_lo = p.window > 0 ? s.first + i - p.window + 1 : 0;
    const long long row = (long long)(s.c0 + i) * p.Hq + hq;
    // positions that the workgroup and this wave hold
    const int t_lo = s.first + f0 / G, t_hi = min(s.first + min(flat - 1, f0 + kTileRows - 1) / G, s.len - 1);
    const int w_lo = min(s.first + wf0 / G, s.len - 1), w_hi = s.first + min(flat - 1, wf0 + 31) / G;

    const KeyBlocks kb = key_blocks<kBlk>(t_lo, t_hi, p.window, p.sinks);
    const int per = (kb.n + p.nsplit - 1) / p.nsplit;
    const int j0 = split * per, j1 = min(kb.n, j0 + per);

    Core core;
    core.init(lds, lane, p.scale);
#pragma unroll
    for (int k = 0; k < Core::kDK; ++k)
        core.qop[k] = *reinterpret_cast<const u32x4*>(p.q + (s.c0 + i) * p.qstride + hq * D + 16 * k + 8 * half);

    const int* trow = p.table + (long long)b * p.table_width;
    const int lp = p.c.lpage, page_mask = (1 << lp) - 1;
    auto page_of = [&](int key) { return trow[min(key >> lp, p.table_width - 1)]; };
    auto no_page = [&](int page) { return (unsigned)page >= (unsigned)p.c.num_pages; };
    // Whether some key that a row here may see has no page (then scores and V
    // are masked by the table too)
    bool holes = false;
    {
        for (int k = (kb.lo >> lp) + tid; k <= t_hi >> lp; k += 64 * NW) holes |= no_page(page_of(k << lp));
        const int ns = min(min(p.sinks, kb.lo), t_hi + 1);
        for (int k = tid; k << lp < ns; k += 64 * NW) holes |= no_page(page_of(k << lp));
    }
    {
        // (through the tiles' LDS: static LDS would take the room of a second
        // workgroup)
        uint32_t* flags = reinterpret_cast<uint32_t*>(lds);
        const bool mine = __any(holes);
        if (lane == 0) flags[wave] = mine;
        __syncthreads();
        uint32_t any = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) any |= flags[w];
        holes = __builtin_amdgcn_readfirstlane(any);
        __syncthreads();
    }

    // A thread's pieces of a block's codes, c = tid, tid + threads, ..: of K row
    // c / (D/16), elements 16 (c % (D/16)) ..; of V the 16-token group c / D,
    // element c % D.  K comes in pairs of half blocks of 32 keys: the upper one
    // of block jj and the lower one of block jj + 1.  All that depends on the
    // thread is in a constant offset, all that depends on the block is uniform
    // in the wave.
    constexpr int kThreads = 64 * NW;
    u32x4 kraw[kPer], vraw[kPer];
    uint32_t ke[kPer], ve[kPer];
    int kpage[kPer], vpage[kPer];
    const uint32_t page_bytes = (uint32_t)D << lp;
    uint32_t kin[kPer], vin[kPer];                              // byte offsets inside a page
    uint32_t kst[kPer], vst[kPer];                              // and inside an LDS tile
    int kup[kPer];                                              // the piece's half block of the pair (uniform)
    int kslot[kPer], vslot[kPer];                               // table entries behind the half block's / block's first
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int c = (tid + u * kThreads) % kChunks;           // (D = 64, eight waves: two threads per piece)
        const int kr = c / (D / 16), kc = c % (D / 16), r = kr & 31, vg = c / D, vd = c % D;
        const int kx = D == 128 ? (r & 15) : ((r >> 1) & 7), vx = (vd >> 1) & 7;
        kup[u] = __builtin_amdgcn_readfirstlane(kr >> 5);
        kslot[u] = r >> lp;
        vslot[u] = 16 * vg >> lp;
        kin[u] = (r & page_mask) * D + 16 * kc;
        vin[u] = (16 * vg & page_mask) * D + 16 * vd;
        kst[u] = r * 2 * D + 16 * ((2 * kc) ^ kx);
        vst[u] = vd * 2 * kBlk + 16 * ((2 * vg) ^ vx);
    }
    auto k_first = [&](int jj, int u) {                         // the first key of the piece's half block
        return kup[u] ? kb.block(min(jj + 1, j1 - 1)) * kBlk : kb.block(max(jj, j0)) * kBlk + 32;
    };
    // The page of a piece is looked up one step ahead of its codes, so that no
    // load waits for the table.
    auto look_k = [&](int jj) {
#pragma unroll
        for (int u = 0; u < kPer; ++u) kpage[u] = trow[(uint32_t)min((k_first(jj, u) >> lp) + kslot[u], p.table_width - 1)];
    };
    auto look_v = [&](int jj) {
#pragma unroll
        for (int u = 0; u < kPer; ++u) vpage[u] = trow[(uint32_t)min((kb.block(jj) * kBlk >> lp) + vslot[u], p.table_width - 1)];
    };
    // (a page that is none is read as the last one, and masked)
    auto page_head = [&](int page) { return min((uint32_t)page, (uint32_t)p.c.num_pages - 1u) * (uint32_t)p.c.Hkv + (uint32_t)h; };
    auto fetch_k = [&](int jj) {
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const uint32_t ph = page_head(kpage[u]);
            const uint8_t* at = p.c.k + (k_first(jj, u) & page_mask) * D;
            kraw[u] = *reinterpret_cast<const u32x4*>(at + ((uint64_t)ph * page_bytes + kin[u]));
            ke[u] = p.c.ke[ph];
        }
    };
    auto fetch_v = [&](int jj) {
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const uint32_t ph = page_head(vpage[u]);
            const uint8_t* at = p.c.v + (kb.block(jj) * kBlk & page_mask) * D;
            vraw[u] = *reinterpret_cast<const u32x4*>(at + ((uint64_t)ph * page_bytes + vin[u]));
            ve[u] = p.c.ve[ph];
        }
    };
    // V's codes of keys that no row here sees (behind the last, in front of the
    // window, a missing page) become zeros
    auto clean_v = [&](int jj) {
        const int key0 = kb.block(jj) * kBlk;
        if (key0 + kBlk - 1 <= t_hi && (key0 >= kb.lo || key0 + kBlk <= p.sinks) && !holes) return;
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int k0 = key0 + (tid + u * kThreads) % kChunks / D * 16;
            const uint32_t seen = keys_seen(k0, t_hi, kb.lo, p.sinks, no_page(page_of(k0)));
#pragma unroll
            for (int w = 0; w < 4; ++w) vraw[u][w] &= byte_mask(seen, w);
        }
    };
    auto store_k = [&](int slot) {                              // the pair into slots slot and (slot + 1) % 4
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const uint32_t at = kst[u] + ((slot + kup[u]) & 3) * kHalf;
            const float s = pow2_of_byte(ke[u]);
            *reinterpret_cast<u32x4*>(lds + at) = dequant8(kraw[u][0], kraw[u][1], s);
            *reinterpret_cast<u32x4*>(lds + (at ^ 16)) = dequant8(kraw[u][2], kraw[u][3], s);
        }
    };
    auto store_v = [&](int buf) {                               // buf: byte offset of the block
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const uint32_t at = vst[u] + buf;
            const float s = pow2_of_byte(ve[u]);
            *reinterpret_cast<u32x4*>(lds + at) = dequant8(vraw[u][0], vraw[u][1], s);
            *reinterpret_cast<u32x4*>(lds + (at ^ 16)) = dequant8(vraw[u][2], vraw[u][3], s);
        }
    };

    const float ninf = -__builtin_huge_valf();
    // masks 32 keys' scores
    auto settle = [&](f32x16& sc, int key0, auto first) {
        if (key0 + 31 > w_lo || (p.window > 0 && key0 <= w_hi - p.window && key0 + 32 > p.sinks) || holes) {
            const int k0 = key0 + Core::kKeyHalf * half;
            const int hi = pos - k0, lo = win_lo - k0, snk = p.sinks - k0;
            const bool gone0 = holes && no_page(page_of(key0)), gone1 = holes && no_page(page_of(key0 + 16));
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int k = Core::key_of(r);
                sc[r] = (k <= hi) & ((k >= lo) | (k < snk)) & !(r < 8 ? gone0 : gone1) ? sc[r] : ninf;
            }
        }
        core.template settle<decltype(first)::value>(sc);
    };

    // The scores of the next 32 keys are formed while those of the current 32
    // turn into P: the matrix unit and the VALU work on independent values.  In
    // step j LDS holds the halves 2 j + 1 and 2 j + 2 of K and V of blocks j - 1
    // and j; 2 j + 3, 2 j + 4 and V of j + 1 come in.
    f32x16 sa, sb;
    uint32_t vcur = kVBase, vnext = Core::next_v(kVBase);
    auto step = [&](auto par_, int j) {
        constexpr int par = decltype(par_)::value, s1 = 2 * par + 1, s2 = (2 * par + 2) & 3;   // par: (j - j0) & 1
        const bool more = j + 1 < j1;
        __syncthreads();
        if (more) clean_v(j + 1);
        __builtin_amdgcn_s_setprio(1);                          // (the other wave of the SIMD settles meanwhile)
        core.fused(sa, sb, s1, vcur, 0);
        __builtin_amdgcn_s_setprio(0);
        settle(sb, kb.block(j) * kBlk + 32, std::false_type{});
        if (more) {
            store_v(vnext);
            if (j + 2 < j1) {
                fetch_v(j + 2);
                if (j + 3 < j1) look_v(j + 3);
            }
        }
        __builtin_amdgcn_s_setprio(1);
        core.fused(sb, sa, s2, vcur, 1);                             // (past the last block: scores that nobody reads)
        __builtin_amdgcn_s_setprio(0);
        if (more) {
            settle(sa, kb.block(j + 1) * kBlk, std::false_type{});
            store_k((s1 + 2) & 3);
            if (j + 2 < j1) {
                fetch_k(j + 2);
                if (j + 3 < j1) look_k(j + 3);
            }
        }
        vcur = vnext;
        vnext = Core::next_v(vnext);
    };
    if (j0 < j1) {
        look_k(j0 - 1);
        look_v(j0);
        fetch_k(j0 - 1);
        fetch_v(j0);
        look_k(j0);
        if (j0 + 1 < j1) look_v(j0 + 1);
        store_k(3);                                             // (slot 3: unused) and half 0 into slot 0
        fetch_k(j0);
        if (j0 + 1 < j1) look_k(j0 + 1);
        clean_v(j0);
        store_v(kVBase);
        if (j0 + 1 < j1) {
            fetch_v(j0 + 1);
            if (j0 + 2 < j1) look_v(j0 + 2);
        }
        store_k(1);
        if (j0 + 1 < j1) {
            fetch_k(j0 + 1);
            if (j0 + 2 < j1) look_k(j0 + 2);
        }
        __syncthreads();
        core.first(sa, 0);
        settle(sa, kb.block(j0) * kBlk, std::true_type{});
        for (int j = j0; j < j1; j += 2) {
            step(std::integral_constant<int, 0>{}, j);
            if (j + 1 < j1) step(std::integral_constant<int, 1>{}, j + 1);
        }
        core.finish();
    }
    const float l = core.total(), m = core.m;
    if (!row_ok) return;
    if (p.nsplit > 1) {
        const long long at = (long long)split * p.total_q * p.Hq + row;
#pragma unroll
        for (int t = 0; t < Core::kDT; ++t)
#pragma unroll
            for (int q = 0; q < 4; ++q) *reinterpret_cast<f32x4*>(p.part + at * D + 32 * t + 8 * q + 4 * half) = core.out4(t, q, 1.0f);
        if (half == 0) {
            p.ml[2 * at] = m;
            p.ml[2 * at + 1] = l;
        }
        return;
    }
    const bool empty = m == ninf;
    const float inv = empty ? 0.0f : 1.0f / l;
#pragma unroll
    for (int t = 0; t < Core::kDT; ++t)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4 v = core.out4(t, q, inv);
            *reinterpret_cast<u32x2*>(p.o + row * D + 32 * t + 8 * q + 4 * half) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        }
    if (p.lse && half == 0) p.lse[row] = empty ? ninf : 0.69314718055994531f * (m + log2f(l));
}

// ---------------------------------------------------------------- combine
// One workgroup per (sequence, row, head); rows that belong to no sequence are
// none of them and stay as they are.
template <int D>
__global__ __launch_bounds__(256) void baps_cache_combine_kernel(CacheAttnParams p)
{
    const int hq = blockIdx.x % p.Hq, i = blockIdx.x / p.Hq % p.max_q, b = blockIdx.x / p.Hq / p.max_q;
    const Seq s = sequence(p, b);
    if (i >= s.n) return;
    const long long row = (long long)(s.c0 + i) * p.Hq + hq;
    f32x4 o;
    float lse;
    if (!combine_row<D>(p.part, p.ml, p.nsplit, (long long)p.total_q * p.Hq, row, o, lse)) return;
    *reinterpret_cast<u32x2*>(p.o + row * D + 4 * threadIdx.x) = u32x2{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
    if (p.lse && threadIdx.x == 0) p.lse[row] = lse;
}

// The same for up to kFewSplits parts, 1024 / D rows per workgroup.
template <int D>
__global__ __launch_bounds__(256) void baps_cache_combine_few_kernel(CacheAttnParams p)
{
    const long long at = (long long)blockIdx.x * (1024 / D) + threadIdx.x / (D / 4);
    const int d4 = threadIdx.x % (D / 4);
    const int hq = (int)(at % p.Hq), i = (int)(at / p.Hq % p.max_q), b = (int)(at / p.Hq / p.max_q);
    if (b >= p.B) return;
    const Seq s = sequence(p, b);
    if (i >= s.n) return;
    const long long row = (long long)(s.c0 + i) * p.Hq + hq;
    f32x4 o;
    float lse;
    combine_row_few<D>(p.part, p.ml, p.nsplit, (long long)p.total_q * p.Hq, row, d4, o, lse);
    *reinterpret_cast<u32x2*>(p.o + row * D + 4 * d4) = u32x2{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
    if (p.lse && d4 == 0) p.lse[row] = lse;
}

// Up to this many flattened rows per key/value head go to the rows kernel, 16 or
// 32 per workgroup
constexpr long long kFewRows = 64;
int few_rows_tile(long long flat) { return flat <= kRows ? kRows : 2 * kRows; }
// Waves of 32 rows in a workgroup of the tile kernel.  Four, with two workgroups per
// CU that fill each other's starts and ends (D = 64: 156 -> 147 us for four sequences
// of 3000 to 4000 keys, 16 heads; D = 128: four of 256 new on 1024 keys 42 -> 36); but
// at D = 128 eight past 1536 keys, for codes are turned to bf16 half as often (2048
// new on 32768 keys 1109 -> 994, 512 on 9000 99 -> 91).
int tile_waves(int D, int max_len, int window, int sinks)
{
    const long long reach = (long long)window + sinks;
    return D == 64 || (window > 0 && reach < max_len ? reach : max_len) <= 1536 ? 4 : 8;
}

template <int D, int NW>
hipError_t launch_tile(const CacheAttnParams& p, long long flat, hipStream_t st)
{
    static DeviceOnce attr_set;
    const int bytes = TileCore<D, false>::kLds;
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (!attr_set.is_done(dev)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(&baps_cache_tile_kernel<D, NW>),
                                hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
        attr_set.mark(dev);
    }
    const long long tiles = (flat + 32 * NW - 1) / (32 * NW);
    hipLaunchKernelGGL((baps_cache_tile_kernel<D, NW>), dim3((unsigned)(tiles * p.B * p.c.Hkv * p.nsplit)), dim3(64 * NW), bytes,
                       st, p);
    return hipGetLastError();
}

template <int D>
hipError_t launch_d(const CacheAttnParams& p, hipStream_t st)
{
    const long long flat = (long long)p.max_q * (p.Hq / p.c.Hkv);
    if (flat <= kFewRows) {
        const int rows = few_rows_tile(flat);
        const dim3 grid((unsigned)p.nsplit, (unsigned)((flat + rows - 1) / rows * p.c.Hkv), (unsigned)p.B), wg(64 * kWaves);
        if (rows > kRows) hipLaunchKernelGGL((baps_cache_rows_kernel<D, 2, false>), grid, wg, 0, st, p);
        else if (p.once) hipLaunchKernelGGL((baps_cache_rows_kernel<D, 1, true>), grid, wg, 0, st, p);
        else hipLaunchKernelGGL((baps_cache_rows_kernel<D, 1, false>), grid, wg, 0, st, p);
    } else {
        hipError_t e = hipSuccess;
        if constexpr (D == 128)
            e = tile_waves(D, p.max_len, p.window, p.sinks) == 8 ? launch_tile<128, 8>(p, flat, st) : launch_tile<128, 4>(p, flat, st);
        else
            e = launch_tile<64, 4>(p, flat, st);
        if (e != hipSuccess) return e;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.nsplit == 1) return e;
    const long long rows = (long long)p.B * p.max_q * p.Hq;
    if (p.nsplit <= kFewSplits)
        hipLaunchKernelGGL((baps_cache_combine_few_kernel<D>), dim3((unsigned)((rows + 1024 / D - 1) / (1024 / D))), dim3(256), 0, st, p);
    else
        hipLaunchKernelGGL((baps_cache_combine_kernel<D>), dim3((unsigned)rows), dim3(256), 0, st, p);
    return hipGetLastError();
}

}  // namespace

// The time of n splits of the tile kernel's keys, in us beyond what any call takes:
// the 64-key blocks of a workgroup in turn, or all of them over the workgroups that
// run at once, and the join: a launch, and the parts written and read.  avg: blocks
// per tile over a chunk, whose first rows see fewer.  (1024 keys, 256 new: 28 us with
// two splits, 22 with four, 20 with eight; 32 heads over 8 of 3800, 1850 new, D =
// 128: 115 whole, 121 with two; 32 over 8 of 9000, 512 new, D = 64: 94 with two, 67
// with four, 64 with six.)
double tile_time(int n, int D, int waves, double blocks, double avg, double groups, double rows, int ncu)
{
    const double step = D == 128 ? 2.0 : 1.4, at_once = waves == 8 ? ncu : 2.0 * ncu;
    const double longest = blocks / n, shared = groups * avg / at_once;
    return step * (longest > shared ? longest : shared) + (n > 1 ? 6.0 + rows * n * 8 * D / 5e6 : 0.0);
}

// The same of the rows kernel where its workgroups are more than the CUs: a CU takes
// 25 GB/s of codes, whether one or two workgroups read them, so the one with most
// sets the time (40 sequences of 6600 keys, 320 workgroups: 120 us, 102, 95 and 94
// with two, three and four splits; 64 of them, 512 workgroups: 141, 144, 145, 148.
// At D = 64, where more workgroups share a CU, 400 of them take 62 whole, 77, 64 and
// 72.)
double rows_time(int n, int D, double keys, long long groups, double rows, int ncu)
{
    const long long of_a_cu = (groups * n + ncu - 1) / ncu;
    return of_a_cu * keys / n * 2 * D / 25e3 * (1 + 0.02 * (n - 1)) + (n > 1 ? 4.0 + rows * n * 8 * D / 5e6 : 0.0);
}

int cache_attention_splits(int B, int Hq, int Hkv, int D, int total_q, int max_q, int max_len, int window, int sinks, int ncu)
{
    const long long flat = (long long)max_q * (Hq / Hkv);
    const bool few = flat <= kFewRows;
    const int waves = tile_waves(D, max_len, window, sinks), rows = few ? few_rows_tile(flat) : 32 * waves;
    // (ragged chunks: no more tiles than all rows fill, and one more each)
    const long long groups = Hkv * std::min((flat + rows - 1) / rows * B, (long long)total_q * (Hq / Hkv) / rows + B);
    long long keys = max_len;                                   // that a workgroup's rows reach
    const long long held = few ? max_q : rows / (Hq / Hkv) + 1, span = (long long)window + sinks + held + 2 * kStep;
    if (window > 0 && span < keys) keys = span;
    const long long blocks = (keys + kStep - 1) / kStep;
    if (few) {
        const int most = (int)std::min(blocks / (2 * kWaves), (long long)kMaxSplits);   // two steps per wave and split at least
        if (groups <= ncu) return std::max(std::min((int)(2 * ncu / groups), most), 1);
        int best = 1;
        double least = 0.9 * rows_time(1, D, keys, groups, 0, ncu);
        for (int n = 2; D == 128 && n <= std::min(most, kFewSplits); ++n) {
            const double t = rows_time(n, D, keys, groups, (double)total_q * Hq, ncu);
            if (t < least) {
                least = t;
                best = n;
            }
        }
        return best;
    }
    const double avg = window > 0 ? (double)blocks : std::max((double)blocks - max_q / 128.0, blocks / 2.0);
    const double whole = tile_time(1, D, waves, blocks, avg, groups, (double)total_q * Hq, ncu);
    int best = 1;
    double least = 0.9 * whole;                                 // (a split is to gain a tenth)
    for (int n = 2; n <= kMaxSplits && n <= blocks; ++n) {
        const double t = tile_time(n, D, waves, blocks, avg, groups, (double)total_q * Hq, ncu);
        if (t < least) {
            least = t;
            best = n;
        }
    }
    return best;
}

hipError_t launch_cache_attention(const CacheAttnParams& p, int D, hipStream_t st)
{
    return D == 64 ? launch_d<64>(p, st) : launch_d<128>(p, st);
}

}  // namespace baps
