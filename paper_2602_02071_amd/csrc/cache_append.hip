// New tokens into the paged 8-bit cache.
//
// One workgroup per (sequence, page that the new tokens touch, key/value head,
// K or V): the scale is that of the whole page, so the page is the unit of the
// maximum.  e is the least exponent with amax <= 448 * 2^(e-127) over the new
// tokens of the page, and no less than what the page has when it holds earlier
// tokens; where it rises those are moved to the new scale (code * 2^(old - e),
// rounded once more).  bf16 -> fp32 and the scaling by a power of two are
// exact, so a code is one rounding (to nearest even) from its value.
//
// A thread holds units of 4 tokens x 8 elements: four 16-byte loads, and
// either four 8-byte stores (K) or eight 4-byte words into LDS that make up
// V's [16 tokens] transposed groups, which leave as 16-byte stores.  The words
// go in 144-byte blocks of eight d's (128 and one 16-byte gap), which puts the
// 64 lanes of a store on 64 banks.  Bound by memory: eight prompts of 2100 to 6500
// tokens, 8 heads, D = 128, 33 us, 5.6 TB/s, as a copy of as many bytes.
#include "cache.hpp"

namespace baps {

namespace {

template <int D, int PAGE>
struct ACfg {
    static constexpr int kUnits = PAGE * D / 32;                // units of 4 tokens x 8 elements
    static constexpr int kThreads = kUnits < 64 ? 64 : (kUnits > 256 ? 256 : kUnits);
    static constexpr int kPer = (kUnits + kThreads - 1) / kThreads;
};

__device__ __forceinline__ float pow2_of_byte(int e) { return hif8::u2f((uint32_t)e << 23); }

// four fp32 values, already scaled, as four codes (saturating, NaN stays NaN)
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d)
{
    auto sat = [](float x) { return x != x ? x : __builtin_amdgcn_fmed3f(x, -448.0f, 448.0f); };
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(sat(a), sat(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(sat(c), sat(d), w, true);
}

__device__ __forceinline__ uint32_t byte_of(uint32_t w, int i) { return (w >> (8 * i)) & 0xffu; }

// four codes moved by a factor 2^-k
__device__ __forceinline__ uint32_t moved4(uint32_t w, float f)
{
    return codes4(__builtin_amdgcn_cvt_f32_fp8(w, 0) * f, __builtin_amdgcn_cvt_f32_fp8(w, 1) * f,
                  __builtin_amdgcn_cvt_f32_fp8(w, 2) * f, __builtin_amdgcn_cvt_f32_fp8(w, 3) * f);
}

// 4 x 4 bytes transposed: out[i] holds byte i of w[0..3]
__device__ __forceinline__ void transpose4(const uint32_t (&w)[4], uint32_t (&out)[4])
{
    const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u);   // w0.0 w1.0 w0.1 w1.1
    const uint32_t b = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);
    const uint32_t c = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);   // w0.2 w1.2 w0.3 w1.3
    const uint32_t d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
    out[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
    out[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
    out[2] = __builtin_amdgcn_perm(d, c, 0x05040100u);
    out[3] = __builtin_amdgcn_perm(d, c, 0x07060302u);
}

template <int D, int PAGE>
__global__ __launch_bounds__((ACfg<D, PAGE>::kThreads)) void baps_cache_append_kernel(CacheAppendParams p)
{
    using C = ACfg<D, PAGE>;
    constexpr int kCh = D / 8;                                  // 8-element chunks of a row
    __shared__ uint32_t wmax[4];
    __shared__ __attribute__((aligned(16))) uint8_t vt[PAGE * D / 8 * 9];
    const int tid = threadIdx.x;
    const int h = blockIdx.y >> 1;
    const bool is_v = blockIdx.y & 1;
    const int slots = gridDim.x / p.B;
    const int b = blockIdx.x / slots;

    // every value that comes from the caller's arrays is held to its range
    // before it forms an address
    const int c0 = p.cu[b], c1 = p.cu[b + 1];
    if (c0 < 0 || c1 <= c0 || c1 > p.total) return;
    const int n = c1 - c0;
    const int len = (int)min((long long)p.lens[b], (long long)p.table_width * PAGE);
    if (p.lens[b] < n) return;
    const int start = p.lens[b] - n;
    const int slot = start / PAGE + blockIdx.x % slots;
    if (slot >= p.table_width) return;
    const int base = slot * PAGE;
    if (base >= len) return;
    const int page = p.table[(long long)b * p.table_width + slot];
    if (page < 0 || page >= p.c.num_pages) return;
    const int held = max(0, start - base);                      // tokens [0, held) of the page are older,
    const int end = min(PAGE, len - base);                      // [held, end) new

    const uint16_t* src = is_v ? p.v : p.k;
    const long long ph = (long long)page * p.c.Hkv + h;
    uint8_t* dst = (is_v ? p.c.v : p.c.k) + ph * (PAGE * D);
    uint8_t* exps = (is_v ? p.c.ve : p.c.ke) + ph;
    const int e_old = held > 0 ? min((int)*exps, kCacheExpHi) : 0;

    u32x4 x[C::kPer][4];
    uint32_t amax = 0;
#pragma unroll
    for (int u = 0; u < C::kPer; ++u) {
        const int unit = tid + u * C::kThreads;
        const int ch = unit % kCh, r0 = unit / kCh * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = r0 + i;
            x[u][i] = u32x4{0, 0, 0, 0};
            if (r >= held && r < end)
                x[u][i] = *reinterpret_cast<const u32x4*>(src + (long long)(c0 + base + r - start) * p.stride + h * D + ch * 8);
#pragma unroll
            for (int w = 0; w < 4; ++w)
#pragma unroll
                for (int s = 0; s < 32; s += 16) {
                    const uint32_t a = (x[u][i][w] >> s) & 0x7fffu;
                    amax = max(amax, a > 0x7f80u ? 0u : a);     // (a NaN sets no scale)
                }
        }
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) amax = max(amax, (uint32_t)__shfl_xor((int)amax, o, 64));
    if ((tid & 63) == 0) wmax[tid >> 6] = amax;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < C::kThreads / 64; ++w) amax = max(amax, wmax[w]);
    // amax = 2^(E-127) (1 + m/128) against 448 = 1.75 * 2^8
    int e = (int)(amax >> 7) - 8 + ((amax & 0x7fu) > 96u ? 1 : 0);
    e = max(e_old, min(max(e, kCacheExpLo), kCacheExpHi));
    const bool moves = held > 0 && e > e_old;
    const float inv = pow2_of_byte(254 - e);                    // 2^(127 - e)
    const float back = moves ? hif8::u2f((uint32_t)max(127 + e_old - e, 0) << 23) : 1.0f;   // (0 below 2^-126: every code is)
    if (tid == 0) *exps = (uint8_t)e;
    const int wlo = moves ? 0 : held;                           // tokens [wlo, end) are written

#pragma unroll
    for (int u = 0; u < C::kPer; ++u) {
        const int unit = tid + u * C::kThreads;
        const int ch = unit % kCh, r0 = unit / kCh * 4;
        if (C::kUnits < 64 && unit >= C::kUnits) break;
        uint32_t lo[4], hi[4];                                  // per token: elements 0..3 and 4..7
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const u32x4 w = x[u][i];
            auto f = [&](int k) {
                return hif8::u2f((k & 1) ? (w[k >> 1] & 0xffff0000u) : (w[k >> 1] << 16)) * inv;
            };
            lo[i] = codes4(f(0), f(1), f(2), f(3));
            hi[i] = codes4(f(4), f(5), f(6), f(7));
        }
        if (!is_v) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = r0 + i;
                uint8_t* at = dst + r * D + ch * 8;
                if (r >= held && r < end) {
                    *reinterpret_cast<u32x2*>(at) = u32x2{lo[i], hi[i]};
                } else if (moves && r < held) {
                    const u32x2 old = *reinterpret_cast<const u32x2*>(at);
                    *reinterpret_cast<u32x2*>(at) = u32x2{moved4(old[0], back), moved4(old[1], back)};
                }
            }
        } else {
            uint32_t t[8];
            transpose4(lo, *reinterpret_cast<uint32_t(*)[4]>(t));
            transpose4(hi, *reinterpret_cast<uint32_t(*)[4]>(t + 4));
            uint8_t* at = vt + (r0 >> 4) * (D * 18) + ch * 144 + (r0 & 15);
#pragma unroll
            for (int k = 0; k < 8; ++k) *reinterpret_cast<uint32_t*>(at + k * 16) = t[k];
        }
    }
    if (!is_v) return;
    __syncthreads();
    // groups of 16 tokens: whole ones are stored as they are, others keep
    // the bytes of the tokens that are not written
    for (int i = tid; i < PAGE / 16 * D; i += C::kThreads) {
        const int g = i / D, d = i % D;
        const int a = max(wlo - 16 * g, 0), z = min(end - 16 * g, 16);
        if (z <= a) continue;
        const u32x4 now = *reinterpret_cast<const u32x4*>(vt + g * (D * 18) + (d >> 3) * 144 + (d & 7) * 16);
        u32x4* at = reinterpret_cast<u32x4*>(dst + (long long)i * 16);
        if (a == 0 && z == 16 && held <= 16 * g) {
            *at = now;
            continue;
        }
        const u32x4 old = *at;
        u32x4 out;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const uint32_t mv = moves ? moved4(old[w], back) : old[w];
            uint32_t r = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = 16 * g + 4 * w + k;               // token of the page
                const uint32_t pick = t >= end ? old[w] : (t >= held ? now[w] : mv);
                r |= pick & (0xffu << (8 * k));
            }
            out[w] = r;
        }
        *at = out;
    }
}

template <int D, int PAGE>
hipError_t launch_append(const CacheAppendParams& p, hipStream_t st)
{
    const long long slots = ((long long)p.max_new + 2 * PAGE - 2) / PAGE;
    hipLaunchKernelGGL((baps_cache_append_kernel<D, PAGE>), dim3((unsigned)(slots * p.B), (unsigned)(2 * p.c.Hkv)),
                       dim3(ACfg<D, PAGE>::kThreads), 0, st, p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_append(const CacheAppendParams& p, int D, hipStream_t st)
{
    switch ((D == 128 ? 8 : 0) + p.c.lpage) {
    case 4: return launch_append<64, 16>(p, st);
    case 5: return launch_append<64, 32>(p, st);
    case 6: return launch_append<64, 64>(p, st);
    case 7: return launch_append<64, 128>(p, st);
    case 12: return launch_append<128, 16>(p, st);
    case 13: return launch_append<128, 32>(p, st);
    case 14: return launch_append<128, 64>(p, st);
    case 15: return launch_append<128, 128>(p, st);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace baps
