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
// bytes.  tile: 256 rows per workgroup, for chunks of a prompt; bound by the
// matrix unit and the exponentials.  Either splits the keys of a row over
// workgroups where rows alone are too few, and combine joins the parts.
#include "cache.hpp"

namespace baps {

namespace {

typedef __bf16 bf16x2 __attribute__((__vector_size__(2 * sizeof(__bf16))));
typedef __bf16 bf16x2e __attribute__((ext_vector_type(2)));

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

// eight codes (two words) times 2^(e-127), e given as that power's fp32 value
__device__ __forceinline__ u32x4 dequant8(uint32_t a, uint32_t b, float s)
{
    return u32x4{__builtin_bit_cast(uint32_t, (bf16x2e)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, false)),
                 __builtin_bit_cast(uint32_t, (bf16x2e)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, true)),
                 __builtin_bit_cast(uint32_t, (bf16x2e)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, false)),
                 __builtin_bit_cast(uint32_t, (bf16x2e)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, true))};
}

__device__ __forceinline__ float pow2_of_byte(int e) { return hif8::u2f((uint32_t)e << 23); }

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}

// A sequence's new tokens and length, held to what the buffers have.
struct Seq {
    int c0, n, first, len;          // packed rows [c0, c0 + n) at positions first ..; keys [0, len)
};

__device__ __forceinline__ Seq sequence(const CacheAttnParams& p, int b)
{
    Seq s;
    const int c1 = p.cu[b + 1], len = p.lens[b];
    s.c0 = p.cu[b];
    s.n = c1 - s.c0;
    if (s.c0 < 0 || s.n <= 0 || c1 > p.total_q) s.n = 0;
    s.first = len - s.n;
    s.n = min(s.n, p.max_q);
    s.len = (int)min((long long)len, (long long)p.table_width << p.c.lpage);
    return s;
}

// A 16-token group of the cache: its page's place for one head, and whether
// there is such a page (a missing one is read as page 0 and masked).
struct Group {
    long long ph;                   // page * Hkv + head
    bool bad;
};

__device__ __forceinline__ Group group_at(const CacheAttnParams& p, const int* row, int key, int h)
{
    const int slot = min(key >> p.c.lpage, p.table_width - 1);
    const int page = row[slot];
    Group g;
    g.bad = (unsigned)page >= (unsigned)p.c.num_pages;
    g.ph = (long long)(g.bad ? 0 : page) * p.c.Hkv + h;
    return g;
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
// product is free where the bytes bound the kernel.
constexpr int kStep = 64;
constexpr int kRows = 16;
constexpr int kWaves = 4;

template <int D>
__global__ __launch_bounds__(64 * kWaves, 2) void baps_cache_rows_kernel(CacheAttnParams p)
{
    constexpr int kJ = D / 64;                                  // 16-byte pieces of a K row per lane
    constexpr int kDT = D / 16;                                 // 16-wide d tiles of O^T
    __shared__ float ldo[kWaves - 1][kRows][D];
    __shared__ float ldm[kWaves][kRows], ldl[kWaves][kRows];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int c16 = lane & 15, grp = lane >> 4;
    const int G = p.Hq / p.c.Hkv;
    const int split = blockIdx.x;
    const int h = blockIdx.y % p.c.Hkv, tile = blockIdx.y / p.c.Hkv;
    const int b = blockIdx.z;
    const Seq s = sequence(p, b);
    const int f0 = tile * kRows, flat = s.n * G;
    if (f0 >= flat) return;

    const int f = f0 + c16;
    const bool row_ok = f < flat;
    const int i = (row_ok ? f : f0) / G, hq = h * G + (row_ok ? f : f0) % G;
    const int t_lo = s.first + f0 / G, t_hi = min(s.first + min(flat - 1, f0 + kRows - 1) / G, s.len - 1);
    const int pos = row_ok ? s.first + i : -1;
    const int win_lo = p.window > 0 ? pos - p.window + 1 : 0;
    const long long row = (long long)(s.c0 + i) * p.Hq + hq;

    const KeyBlocks kb = key_blocks<kStep>(t_lo, t_hi, p.window, p.sinks);
    const int per = (kb.n + p.nsplit - 1) / p.nsplit;
    const int j1 = min(kb.n, (split + 1) * per);
    int j = split * per + wave;

    u32x4 qop[2 * kJ];
#pragma unroll
    for (int k = 0; k < 2 * kJ; ++k)
        qop[k] = *reinterpret_cast<const u32x4*>(p.q + (s.c0 + i) * p.qstride + hq * D + 64 * (k >> 1) + 16 * grp + 8 * (k & 1));

    const int* trow = p.table + (long long)b * p.table_width;
    const int page_mask = (1 << p.c.lpage) - 1;
    const float ninf = -__builtin_huge_valf();
    float m = ninf, l = 0.0f;
    f32x4 oacc[kDT];
#pragma unroll
    for (int t = 0; t < kDT; ++t) oacc[t] = f32x4{};

    u32x4 kr[4][kJ], vr[kDT];
    float ks = 1.0f, vs = 1.0f;
    bool bad = false, bad_n = false;
    auto load_k = [&](int jj) {
        const int key = kb.block(jj) * kStep + 16 * (c16 >> 2);
        const Group g = group_at(p, trow, key, h);
        const uint8_t* at = p.c.k + ((g.ph << p.c.lpage) + (key & page_mask) + (c16 & 3)) * D + 16 * grp;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int k = 0; k < kJ; ++k) kr[t][k] = *reinterpret_cast<const u32x4*>(at + 4 * t * D + 64 * k);
        ks = pow2_of_byte(p.c.ke[g.ph]);
    };
    auto load_v = [&](int jj) {
        const int key = kb.block(jj) * kStep + 16 * grp;
        const Group g = group_at(p, trow, key, h);
        const uint8_t* at = p.c.v + ((g.ph << p.c.lpage) + (key & page_mask)) * D + 16 * c16;
#pragma unroll
        for (int t = 0; t < kDT; ++t) vr[t] = *reinterpret_cast<const u32x4*>(at + 256 * t);
        vs = pow2_of_byte(p.c.ve[g.ph]);
        bad_n = g.bad;
    };
    if (j < j1) {
        load_k(j);
        load_v(j);
    }
    for (; j < j1; j += kWaves) {
        const int key0 = kb.block(j) * kStep;
        const bool more = j + kWaves < j1;
        bad = bad_n;
        f32x4 sacc[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            f32x4 a = {};
#pragma unroll
            for (int k = 0; k < kJ; ++k) {
                a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(dequant8(kr[t][k][0], kr[t][k][1], ks)),
                                                            as_bf16x8(qop[2 * k]), a, 0, 0, 0);
                a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(dequant8(kr[t][k][2], kr[t][k][3], ks)),
                                                            as_bf16x8(qop[2 * k + 1]), a, 0, 0, 0);
            }
            sacc[t] = a;
        }
        if (more) load_k(j + kWaves);
        // Steps that some row does not see whole: scores of hidden keys are
        // -inf, whatever their codes are, and V's codes of keys that no row
        // of the tile sees are zero (what lies behind the last token or in
        // front of the window may be anything, 0 * NaN included).
        if (key0 + kStep - 1 > t_lo || (p.window > 0 && key0 <= t_hi - p.window && key0 + kStep > p.sinks) ||
            __any(bad)) {
            // (bitwise conditions: selects and no branches per score)
            const int k0 = key0 + 16 * grp;
            const int hi = bad ? -1 : min(pos, s.len - 1) - k0, lo = win_lo - k0, snk = p.sinks - k0;
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int k = 4 * t + r;
                    sacc[t][r] = (k <= hi) & ((k >= lo) | (k < snk)) ? sacc[t][r] : ninf;
                }
            const uint32_t seen = keys_seen(k0, t_hi, kb.lo, p.sinks, bad);
#pragma unroll
            for (int t = 0; t < kDT; ++t)
#pragma unroll
                for (int w = 0; w < 4; ++w) vr[t][w] &= byte_mask(seen, w);
        }
        float mx = ninf;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) mx = fmaxf(mx, sacc[t][r]);
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(m, mx * p.scale);
        const float nref = m_new == ninf ? 0.0f : -m_new;
        const float fac = m == ninf ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
        if (__any(fac != 1.0f)) {
#pragma unroll
            for (int t = 0; t < kDT; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) oacc[t][r] *= fac;
        }
        l *= fac;
        m = m_new;
        u32x4 hi[2], lo[2];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            float pr[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                pr[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[t][r], p.scale, nref));
                l += pr[r];
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t w = pack_bf16(pr[2 * e], pr[2 * e + 1]);
                hi[t >> 1][2 * (t & 1) + e] = w;
                lo[t >> 1][2 * (t & 1) + e] = pack_bf16(pr[2 * e] - hif8::u2f(w << 16), pr[2 * e + 1] - hif8::u2f(w & 0xffff0000u));
            }
        }
#pragma unroll
        for (int t = 0; t < kDT; ++t) {
            const bf16x8 v0 = as_bf16x8(dequant8(vr[t][0], vr[t][1], vs)), v1 = as_bf16x8(dequant8(vr[t][2], vr[t][3], vs));
            oacc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, as_bf16x8(hi[0]), oacc[t], 0, 0, 0);
            oacc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, as_bf16x8(hi[1]), oacc[t], 0, 0, 0);
            oacc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, as_bf16x8(lo[0]), oacc[t], 0, 0, 0);
            oacc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, as_bf16x8(lo[1]), oacc[t], 0, 0, 0);
        }
        if (more) load_v(j + kWaves);
    }
    // the waves' parts: a common maximum, then one sum in a fixed order
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (grp == 0) ldm[wave][c16] = m;
    __syncthreads();
    float mt = ldm[0][c16];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) mt = fmaxf(mt, ldm[w][c16]);
    const float fac = m == ninf ? 0.0f : __builtin_amdgcn_exp2f(m - mt);
#pragma unroll
    for (int t = 0; t < kDT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) oacc[t][r] *= fac;
    l *= fac;
    if (grp == 0) ldl[wave][c16] = l;
    if (wave > 0) {
#pragma unroll
        for (int t = 0; t < kDT; ++t) *reinterpret_cast<f32x4*>(&ldo[wave - 1][c16][16 * t + 4 * grp]) = oacc[t];
    }
    __syncthreads();
    if (wave > 0 || !row_ok) return;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) {
#pragma unroll
        for (int t = 0; t < kDT; ++t) {
            const f32x4 x = *reinterpret_cast<const f32x4*>(&ldo[w - 1][c16][16 * t + 4 * grp]);
#pragma unroll
            for (int r = 0; r < 4; ++r) oacc[t][r] += x[r];
        }
        l += ldl[w][c16];
    }
    if (p.nsplit > 1) {
        const long long at = (long long)split * p.total_q * p.Hq + row;
#pragma unroll
        for (int t = 0; t < kDT; ++t) *reinterpret_cast<f32x4*>(p.part + at * D + 16 * t + 4 * grp) = oacc[t];
        if (grp == 0) {
            p.ml[2 * at] = mt;
            p.ml[2 * at + 1] = l;
        }
        return;
    }
    const bool empty = mt == ninf;
    const float inv = empty ? 0.0f : 1.0f / l;
#pragma unroll
    for (int t = 0; t < kDT; ++t)
        *reinterpret_cast<u32x2*>(p.o + row * D + 16 * t + 4 * grp) =
            u32x2{pack_bf16(oacc[t][0] * inv, oacc[t][1] * inv), pack_bf16(oacc[t][2] * inv, oacc[t][3] * inv)};
    if (p.lse && grp == 0) p.lse[row] = empty ? ninf : 0.69314718055994531f * (mt + log2f(l));
}

// ---------------------------------------------------------------- tile kernel
// Eight waves of 32 rows each, blocks of 64 keys.  The codes of a block come
// through registers (one 16-byte load of K and of V per thread at D = 128),
// are dequantised once for the eight waves and stored to LDS as bf16, into a
// double buffer: the loads of block j+2 are in flight and block j+1 is stored
// while block j is computed.  K lies as [key][d], V as [d][key], both with
// their 16-byte chunks XOR-swizzled.  S^T = K Q^T on 32x32x16 with the rows of
// K taken in the order that gives a lane 8 consecutive keys per 16-key chunk
// (row 8a + 4 half + b of the tile is key 16 (a/2) + 8 half + 4 (a%2) + b), so
// V^T's operand is one 16-byte read.
constexpr int kBlk = 64;
constexpr int kTileWaves = 8;
constexpr int kTileRows = 32 * kTileWaves;

template <int D>
__global__ __launch_bounds__(64 * kTileWaves, 2) void baps_cache_tile_kernel(CacheAttnParams p)
{
    constexpr int kDK = D / 16, kDT = D / 32, kKT = kBlk / 32;
    constexpr int kKB = kBlk * D * 2;                           // bytes of a K (or V) tile
    constexpr int kChunks = kBlk * D / 16;                      // 16-byte pieces of codes (512 or 256)
    extern __shared__ __attribute__((aligned(1024))) char lds[];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j32 = lane & 31, half = lane >> 5;
    const int G = p.Hq / p.c.Hkv;
    const int ntiles = gridDim.x / p.nsplit;
    const int split = blockIdx.x % p.nsplit;
    const int tile = ntiles - 1 - blockIdx.x / p.nsplit;        // the tiles with the most keys first
    const int h = blockIdx.y, b = blockIdx.z;
    const Seq s = sequence(p, b);
    const int f0 = tile * kTileRows, flat = s.n * G;
    if (f0 >= flat) return;

    const int f = f0 + wave * 32 + j32;
    const bool row_ok = f < flat;
    const int i = (row_ok ? f : f0) / G, hq = h * G + (row_ok ? f : f0) % G;
    const int pos = row_ok ? min(s.first + i, s.len - 1) : -1;
    const int win_lo = (row_ok && p.window > 0) ? s.first + i - p.window + 1 : 0;
    const long long row = (long long)(s.c0 + i) * p.Hq + hq;
    // positions that the workgroup and this wave hold
    const int t_lo = s.first + f0 / G, t_hi = min(s.first + min(flat - 1, f0 + kTileRows - 1) / G, s.len - 1);
    const int wf0 = f0 + wave * 32;
    const bool wave_ok = wf0 < flat;
    const int w_lo = s.first + wf0 / G, w_hi = min(s.first + min(flat - 1, wf0 + 31) / G, s.len - 1);

    const KeyBlocks kb = key_blocks<kBlk>(t_lo, t_hi, p.window, p.sinks);
    const int per = (kb.n + p.nsplit - 1) / p.nsplit;
    const int j0 = split * per, j1 = min(kb.n, j0 + per);

    u32x4 qop[kDK];
#pragma unroll
    for (int k = 0; k < kDK; ++k)
        qop[k] = *reinterpret_cast<const u32x4*>(p.q + (s.c0 + i) * p.qstride + hq * D + 16 * k + 8 * half);

    const int* trow = p.table + (long long)b * p.table_width;
    const int page_mask = (1 << p.c.lpage) - 1;
    // this thread's piece of a block's codes: K row kr_, elements 16 kc_ ..;
    // V's 16-token group vg_, element vd_
    const bool loads = tid < kChunks;
    const int kr_ = tid / (D / 16) % kBlk, kc_ = tid % (D / 16);
    const int vg_ = tid / D % (kBlk / 16), vd_ = tid % D;
    u32x4 kraw = {}, vraw = {};
    float ks = 1.0f, vs = 1.0f;
    bool vbad = false;
    auto fetch = [&](int jj) {
        if (!loads) return;
        const int key0 = kb.block(jj) * kBlk;
        const Group gk = group_at(p, trow, key0 + kr_, h);
        kraw = *reinterpret_cast<const u32x4*>(p.c.k + ((gk.ph << p.c.lpage) + ((key0 + kr_) & page_mask)) * D + 16 * kc_);
        ks = pow2_of_byte(p.c.ke[gk.ph]);
        const int kv = key0 + 16 * vg_;
        const Group gv = group_at(p, trow, kv, h);
        vraw = *reinterpret_cast<const u32x4*>(p.c.v + ((gv.ph << p.c.lpage) + (kv & page_mask)) * D + 16 * vd_);
        vs = pow2_of_byte(p.c.ve[gv.ph]);
        vbad = gv.bad;
    };
    // codes to LDS; V's of keys that no row here sees (behind the last, in
    // front of the window, a missing page) as zeros
    __shared__ __attribute__((aligned(16))) uint32_t badg[2][kBlk / 16];   // 1: the block's 16-token group has no page
    auto store = [&](int jj, int buf) {
        if (!loads) return;
        const int key0 = kb.block(jj) * kBlk;
        char* kt = lds + buf * 2 * kKB;
        char* vt = kt + kKB;
        const int kx = D == 128 ? (kr_ & 15) : ((kr_ >> 1) & 7);
        *reinterpret_cast<u32x4*>(kt + kr_ * 2 * D + 16 * ((2 * kc_) ^ kx)) = dequant8(kraw[0], kraw[1], ks);
        *reinterpret_cast<u32x4*>(kt + kr_ * 2 * D + 16 * ((2 * kc_ + 1) ^ kx)) = dequant8(kraw[2], kraw[3], ks);
        u32x4 v = vraw;
        const int k0 = key0 + 16 * vg_;
        if (k0 + 15 > t_hi || (k0 < kb.lo && k0 + 15 >= p.sinks) || vbad) {
            const uint32_t seen = keys_seen(k0, t_hi, kb.lo, p.sinks, vbad);
#pragma unroll
            for (int w = 0; w < 4; ++w) v[w] &= byte_mask(seen, w);
        }
        const int vx = (vd_ >> 1) & 7;
        *reinterpret_cast<u32x4*>(vt + vd_ * 2 * kBlk + 16 * ((2 * vg_) ^ vx)) = dequant8(v[0], v[1], vs);
        *reinterpret_cast<u32x4*>(vt + vd_ * 2 * kBlk + 16 * ((2 * vg_ + 1) ^ vx)) = dequant8(v[2], v[3], vs);
        if (vd_ == 0) badg[buf][vg_] = vbad;
    };

    const float ninf = -__builtin_huge_valf();
    float m = ninf, l = 0.0f;
    f32x16 oacc[kDT];
#pragma unroll
    for (int t = 0; t < kDT; ++t) oacc[t] = f32x16{};
    // the lane's K rows: row j32 of a tile is key 16 (a/2) + 8 hf + 4 (a%2) + b
    const int ka = j32 >> 3, kh = (j32 >> 2) & 1;
    const int krow = 16 * (ka >> 1) + 8 * kh + 4 * (ka & 1) + (j32 & 3);
    const int kx = D == 128 ? (krow & 15) : ((krow >> 1) & 7);  // (the same for krow + 32)
    const int vx = (j32 >> 1) & 7;                              // (the same for j32 + 32 t)

    if (j0 < j1) {
        fetch(j0);
        store(j0, 0);
        if (j0 + 1 < j1) fetch(j0 + 1);
    }
    for (int j = j0; j < j1; ++j) {
        const int buf = (j - j0) & 1;
        __syncthreads();                                        // block j is in LDS, block j-1 is done with
        const int key0 = kb.block(j) * kBlk;
        const char* kt = lds + buf * 2 * kKB;
        const char* vt = kt + kKB;
        const u32x4 bg = *reinterpret_cast<const u32x4*>(badg[buf]);
        const uint32_t bad = bg[0] | bg[1] << 1 | bg[2] << 2 | bg[3] << 3;
        // a wave whose rows see nothing of the block leaves it
        const bool live = wave_ok && key0 <= w_hi &&
                          (p.window == 0 || key0 + kBlk - 1 > w_lo - p.window || key0 < p.sinks);
        f32x16 sacc[kKT];
        if (live) {
#pragma unroll
            for (int t = 0; t < kKT; ++t) sacc[t] = f32x16{};
#pragma unroll
            for (int k = 0; k < kDK; ++k)
#pragma unroll
                for (int t = 0; t < kKT; ++t) {
                    const u32x4 a = *reinterpret_cast<const u32x4*>(kt + (32 * t + krow) * 2 * D + 16 * ((2 * k + half) ^ kx));
                    sacc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(qop[k]), sacc[t], 0, 0, 0);
                }
        }
        if (j + 1 < j1) {
            store(j + 1, buf ^ 1);
            if (j + 2 < j1) fetch(j + 2);
        }
        if (!live) continue;
        // register 8c + e of tile t is key 32 t + 16 c + 8 half + e
        if (key0 + kBlk - 1 > w_lo || (p.window > 0 && key0 <= w_hi - p.window && key0 + kBlk > p.sinks) || bad || wf0 + 31 >= flat) {
            const int k0 = key0 + 8 * half;
            const int hi = pos - k0, lo = win_lo - k0, snk = p.sinks - k0;
#pragma unroll
            for (int t = 0; t < kKT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int k = 32 * t + 16 * (r >> 3) + (r & 7);
                    const bool gone = (bad >> (2 * t + (r >> 3))) & 1u;
                    sacc[t][r] = (k <= hi) & ((k >= lo) | (k < snk)) & !gone ? sacc[t][r] : ninf;
                }
        }
        float mx = ninf;
#pragma unroll
        for (int t = 0; t < kKT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sacc[t][r]);
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(m, mx * p.scale);
        const float nref = m_new == ninf ? 0.0f : -m_new;
        const float fac = m == ninf ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
        if (__any(fac != 1.0f)) {
#pragma unroll
            for (int t = 0; t < kDT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) oacc[t][r] *= fac;
        }
        l *= fac;
        m = m_new;
#pragma unroll
        for (int t = 0; t < kKT; ++t) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                u32x4 pop;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[t][8 * c + 2 * e], p.scale, nref));
                    const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[t][8 * c + 2 * e + 1], p.scale, nref));
                    l += p0 + p1;
                    pop[e] = pack_bf16(p0, p1);
                }
#pragma unroll
                for (int dt = 0; dt < kDT; ++dt) {
                    const u32x4 a = *reinterpret_cast<const u32x4*>(vt + (32 * dt + j32) * 2 * kBlk + 16 * ((4 * t + 2 * c + half) ^ vx));
                    oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(pop), oacc[dt], 0, 0, 0);
                }
            }
        }
    }
    l += __shfl_xor(l, 32, 64);
    if (!row_ok) return;
    // register r of d tile dt is element 32 dt + 8 (r/4) + 4 half + r%4
    if (p.nsplit > 1) {
        const long long at = (long long)split * p.total_q * p.Hq + row;
#pragma unroll
        for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
            for (int q4 = 0; q4 < 4; ++q4)
                *reinterpret_cast<f32x4*>(p.part + at * D + 32 * dt + 8 * q4 + 4 * half) =
                    f32x4{oacc[dt][4 * q4], oacc[dt][4 * q4 + 1], oacc[dt][4 * q4 + 2], oacc[dt][4 * q4 + 3]};
        if (half == 0) {
            p.ml[2 * at] = m;
            p.ml[2 * at + 1] = l;
        }
        return;
    }
    const bool empty = m == ninf;
    const float inv = empty ? 0.0f : 1.0f / l;
#pragma unroll
    for (int dt = 0; dt < kDT; ++dt)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
            *reinterpret_cast<u32x2*>(p.o + row * D + 32 * dt + 8 * q4 + 4 * half) =
                u32x2{pack_bf16(oacc[dt][4 * q4] * inv, oacc[dt][4 * q4 + 1] * inv),
                      pack_bf16(oacc[dt][4 * q4 + 2] * inv, oacc[dt][4 * q4 + 3] * inv)};
    if (p.lse && half == 0) p.lse[row] = empty ? ninf : 0.69314718055994531f * (m + log2f(l));
}

// ---------------------------------------------------------------- combine
// One row per D/4 lanes: the parts' common maximum, then their weighted sums
// in split order.  Rows that belong to no sequence are left as they are: the
// row's sequence is looked up, because its parts were not written then.
template <int D>
__global__ __launch_bounds__(256) void baps_cache_combine_kernel(CacheAttnParams p)
{
    constexpr int kLanes = D / 4, kPer = 256 / kLanes;
    const long long rows = (long long)p.total_q * p.Hq;
    const long long row = (long long)blockIdx.x * kPer + threadIdx.x / kLanes;
    const int d = threadIdx.x % kLanes * 4;
    if (row >= rows) return;
    const int t = (int)(row / p.Hq);
    int lo = 0, hi = p.B;                                       // the last sequence with cu[b] <= t
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.cu[mid] <= t) lo = mid; else hi = mid;
    }
    const Seq s = sequence(p, lo);
    if (t < s.c0 || t >= s.c0 + s.n) return;
    const float ninf = -__builtin_huge_valf();
    float m = ninf;
    for (int k = 0; k < p.nsplit; ++k) m = fmaxf(m, p.ml[2 * (k * rows + row)]);
    float l = 0.0f;
    f32x4 o = {};
    if (m != ninf) {
        for (int k = 0; k < p.nsplit; ++k) {
            const float mk = p.ml[2 * (k * rows + row)];
            if (mk == ninf) continue;
            const float w = __builtin_amdgcn_exp2f(mk - m);
            l += w * p.ml[2 * (k * rows + row) + 1];
            const f32x4 x = *reinterpret_cast<const f32x4*>(p.part + (k * rows + row) * D + d);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += w * x[e];
        }
    }
    const float inv = m == ninf ? 0.0f : 1.0f / l;
    *reinterpret_cast<u32x2*>(p.o + row * D + d) = u32x2{pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv)};
    if (p.lse && d == 0) p.lse[row] = m == ninf ? ninf : 0.69314718055994531f * (m + log2f(l));
}

// Up to this many flattened rows per key/value head go to the rows kernel
constexpr long long kFewRows = 64;

template <int D>
hipError_t launch_d(const CacheAttnParams& p, hipStream_t st)
{
    const long long flat = (long long)p.max_q * (p.Hq / p.c.Hkv);
    if (flat <= kFewRows) {
        const dim3 grid((unsigned)p.nsplit, (unsigned)((flat + kRows - 1) / kRows * p.c.Hkv), (unsigned)p.B);
        hipLaunchKernelGGL((baps_cache_rows_kernel<D>), grid, dim3(64 * kWaves), 0, st, p);
    } else {
        static DeviceOnce attr_set;
        const int bytes = 4 * kBlk * D * 2;
        int dev = 0;
        hipError_t e = hipGetDevice(&dev);
        if (e != hipSuccess) return e;
        if (!attr_set.is_done(dev)) {
            e = hipFuncSetAttribute(reinterpret_cast<const void*>(&baps_cache_tile_kernel<D>),
                                    hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
            if (e != hipSuccess) return e;
            attr_set.mark(dev);
        }
        const dim3 grid((unsigned)((flat + kTileRows - 1) / kTileRows * p.nsplit), (unsigned)p.c.Hkv, (unsigned)p.B);
        hipLaunchKernelGGL((baps_cache_tile_kernel<D>), grid, dim3(64 * kTileWaves), bytes, st, p);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.nsplit == 1) return e;
    const long long rows = (long long)p.total_q * p.Hq;
    constexpr int kPer = 256 / (D / 4);
    hipLaunchKernelGGL((baps_cache_combine_kernel<D>), dim3((unsigned)((rows + kPer - 1) / kPer)), dim3(256), 0, st, p);
    return hipGetLastError();
}

}  // namespace

int cache_attention_splits(int B, int Hq, int Hkv, int max_q, int max_len, int window, int sinks, int ncu)
{
    const long long flat = (long long)max_q * (Hq / Hkv);
    const bool few = flat <= kFewRows;
    const long long groups = (flat + (few ? kRows : kTileRows) - 1) / (few ? kRows : kTileRows) * Hkv * B;
    long long keys = max_len;                                   // that a workgroup's rows reach
    const long long span = (long long)window + sinks + max_q + 2 * kStep;
    if (window > 0 && span < keys) keys = span;
    const long long blocks = (keys + kStep - 1) / kStep;
    const long long slots = few ? 2LL * ncu : ncu, least = few ? 2 * kWaves : 8;    // blocks per split at least
    long long n = slots / groups;
    if (n > blocks / least) n = blocks / least;
    return (int)(n < 1 ? 1 : (n > 64 ? 64 : n));
}

hipError_t launch_cache_attention(const CacheAttnParams& p, int D, hipStream_t st)
{
    return D == 64 ? launch_d<64>(p, st) : launch_d<128>(p, st);
}

}  // namespace baps
