// Attention with a sliding window and sink tokens in the Default setup (eq. (2)
// in fp32) for many query rows: 32 NW flattened (position, head of the group) rows
// of a key/value head per workgroup, on the inner loop of tile_core.hpp, over the
// key blocks that the rows' windows and the sinks reach.
//
// K and V come by asynchronous loads straight into LDS, a block of V and two half
// blocks of K per step, a step ahead: nothing is left of staging, and the loop is
// bound by its products and exponentials alone (16384 positions, GQA 32/8, D = 128,
// window 4096: 973 us, 0.99 PFLOP/s).  window_form() says which calls come here,
// and when the keys are split over workgroups, whose parts combine joins.
#include <type_traits>

#include "tile_core.hpp"

namespace baps {

namespace {

#define LDS_PTR(T, p) ((__attribute__((address_space(3))) T*)(p))

// One wave-wide asynchronous load of 1 KiB: lane l's 16 bytes at base + off land at
// LDS byte dst + 16 l.  (Assembly, so that the compiler guards no later LDS read
// with a wait for it; the kernel waits itself, before the barrier that publishes
// the tile.)
__device__ __forceinline__ void load_1k(uint32_t off, uint64_t base, uint32_t dst)
{
    asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(dst) : "memory", "m0");
}

__device__ __forceinline__ void load_1k_at(const void* at, uint32_t dst)
{
    asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(at), "s"(dst) : "memory", "m0");
}

__device__ __forceinline__ uint64_t uniform_addr(const void* p)
{
    const uint64_t a = (uint64_t)(uintptr_t)p;
    return ((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32)) << 32) | (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a);
}

template <int D, int NW>
__global__ __launch_bounds__(64 * NW, 2) void baps_attn_window_tile_kernel(AttnParams p)
{
    using Core = TileCore<D, true>;
    constexpr int kTileRows = 32 * NW;
    constexpr int kRowsPerLoad = 512 / D, kHalfLoads = 32 / kRowsPerLoad;   // rows of a 1 KiB load, loads of a half block
    constexpr int kPer = 2 * kHalfLoads / NW;                   // loads per wave of a pair of half blocks, or of V
    static_assert(kPer * NW == 2 * kHalfLoads, "every wave loads alike");
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)LDS_PTR(char, lds);

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j32 = lane & 31, half = lane >> 5;
    const int G = p.Hq / p.Hkv, flat = p.Sq * G, off = p.Sk - p.Sq;
    // head fastest (eight of them, or a multiple: each XCD's L2 holds its own
    // heads' K and V), the last rows first
    const int heads = p.Hkv * p.B, hb = blockIdx.x % heads;
    const int h = hb % p.Hkv, b = hb / p.Hkv;
    const int split = blockIdx.x / heads % p.nsplit;
    const int f0 = ((flat + kTileRows - 1) / kTileRows - 1 - blockIdx.x / heads / p.nsplit) * kTileRows;

    // (lanes behind the last row compute it again, and store nothing)
    const int wf0 = min(f0 + wave * 32, flat - 1), f = min(f0 + wave * 32 + j32, flat - 1);
    const bool row_ok = f0 + wave * 32 + j32 < flat;
    const int r = f / G, hq = h * G + f % G;
    const int pos = r + off, win_lo = pos - p.window + 1;
    const long long row = ((long long)b * p.Hq + hq) * p.Sq + r;
    const int t_lo = f0 / G + off, t_hi = min(flat - 1, f0 + kTileRows - 1) / G + off;
    const int w_lo = wf0 / G + off, w_hi = min(flat - 1, wf0 + 31) / G + off;
    const KeyBlocks kb = key_blocks<kBlk>(t_lo, t_hi, p.window, p.sinks);
    const int per = (kb.n + p.nsplit - 1) / p.nsplit;
    const int j0 = split * per, j1 = min(kb.n, j0 + per);

    Core core;
    core.init(lds, lane, p.c);
#pragma unroll
    for (int k = 0; k < Core::kDK; ++k) core.qop[k] = *reinterpret_cast<const u32x4*>(p.q + row * D + 16 * k + 8 * half);

    // Lane offsets of this wave's loads t = wave, wave + NW, ..: of a pair of half
    // blocks of K (the upper one of block jj and the lower one of block jj + 1) and
    // of a block of V, with the chunks' XOR swizzle on the memory side
    const uint16_t* kbase = p.k + ((long long)b * p.Hkv + h) * p.Sk * D;
    const uint16_t* vbase = p.v + ((long long)b * p.Hkv + h) * p.Sk * D;
    uint32_t kofs[kPer], vofs[kPer];
    int krow[kPer], vrow[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
        const int t = wave + u * NW, c = lane % (D / 8);
        krow[u] = t % kHalfLoads * kRowsPerLoad + lane / (D / 8);
        vrow[u] = t * kRowsPerLoad + lane / (D / 8);
        kofs[u] = krow[u] * 2 * D + 16 * (c ^ (D == 128 ? (krow[u] & 15) : ((krow[u] >> 1) & 7)));
        vofs[u] = vrow[u] * 2 * D + 16 * (c ^ (D == 128 ? 2 * (vrow[u] & 3) : 2 * ((vrow[u] >> 1) & 1)));
    }
    // rows from `first` on; those past the last key are the last key's (finite, masked)
    auto load = [&](const uint16_t* base, int first, int n, uint32_t ofs, int r_, uint32_t dst) {
        if (first + n <= p.Sk) load_1k(ofs, uniform_addr(base + (long long)first * D), dst);
        else load_1k_at(reinterpret_cast<const char*>(base + (long long)min(first + r_, p.Sk - 1) * D) + (ofs - r_ * 2 * D), dst);
    };
    auto load_k = [&](int jj, int slot) {                       // the pair into slots slot and (slot + 1) % 4
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int t = wave + u * NW, up = t / kHalfLoads;
            const int first = up ? kb.block(min(jj + 1, j1 - 1)) * kBlk : kb.block(max(jj, j0)) * kBlk + 32;
            load(kbase, first, 32, kofs[u], krow[u],
                 __builtin_amdgcn_readfirstlane(lds0 + ((slot + up) & 3) * Core::kHalf + t % kHalfLoads * 1024));
        }
    };
    auto load_v = [&](int jj, uint32_t buf) {
#pragma unroll
        for (int u = 0; u < kPer; ++u)
            load(vbase, kb.block(jj) * kBlk, kBlk, vofs[u], vrow[u], __builtin_amdgcn_readfirstlane(lds0 + buf + (wave + u * NW) * 1024));
    };

    const float ninf = -__builtin_huge_valf();
    auto settle = [&](f32x16& sc, int key0, auto first) {
        if (key0 + 31 > w_lo || (key0 <= w_hi - p.window && key0 + 32 > p.sinks)) {
            const int k0 = key0 + Core::kKeyHalf * half;
            const int hi = pos - k0, lo = win_lo - k0, snk = p.sinks - k0;
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                const int k = Core::key_of(x);
                sc[x] = (k <= hi) & ((k >= lo) | (k < snk)) ? sc[x] : ninf;
            }
        }
        core.template settle<decltype(first)::value>(sc);
    };

    // In step j LDS holds the halves 2 j + 1 and 2 j + 2 of K and V of blocks j - 1
    // and j; 2 j + 3, 2 j + 4 and V of j + 1 are on their way.
    f32x16 sa, sb;
    uint32_t vcur = Core::kVBase;
    auto step = [&](auto par_, int j) {
        constexpr int par = decltype(par_)::value, s1 = 2 * par + 1, s2 = (2 * par + 2) & 3;   // par: (j - j0) & 1
        const bool more = j + 1 < j1;
        const int key0 = kb.block(j) * kBlk;
        __builtin_amdgcn_s_waitcnt(0x0F70);                     // this wave's loads have landed (vmcnt 0)
        __syncthreads();
        if (key0 < kb.lo && key0 + kBlk > p.sinks) {
            zero_hidden_v<2 * D>(lds + vcur, key0, kBlk, kb.lo, p.sinks, tid, 64 * NW);
            __syncthreads();
        }
        if (more) {
            load_v(j + 1, Core::next_v(vcur));
            load_k(j + 1, (s1 + 2) & 3);
        }
        __builtin_amdgcn_s_setprio(1);                          // (the other wave of the SIMD settles meanwhile)
        core.fused(sa, sb, s1, vcur, 0);
        __builtin_amdgcn_s_setprio(0);
        settle(sb, key0 + 32, std::false_type{});
        __builtin_amdgcn_s_setprio(1);
        core.fused(sb, sa, s2, vcur, 1);                        // (past the last block: scores that nobody reads)
        __builtin_amdgcn_s_setprio(0);
        if (more) settle(sa, kb.block(j + 1) * kBlk, std::false_type{});
        vcur = Core::next_v(vcur);
    };
    if (j0 < j1) {
        load_k(j0 - 1, 3);                                      // (slot 3: unused) and half 0 into slot 0
        load_v(j0, Core::kVBase);
        load_k(j0, 1);
        __builtin_amdgcn_s_waitcnt(0x0F70);
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
        const long long at = split * ((long long)p.B * p.Hq * p.Sq) + row;
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
            const long long at = row * D + 32 * t + 8 * q + 4 * half;
            if (p.out_bf16) *reinterpret_cast<u32x2*>(reinterpret_cast<uint16_t*>(p.o) + at) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
            else *reinterpret_cast<f32x4*>(p.o + at) = v;
        }
    if (p.lse && half == 0) p.lse[row] = empty ? ninf : 0.69314718055994531f * (m + log2f(l));
}

template <int D, int NW>
hipError_t launch_rows(const AttnParams& p, hipStream_t st)
{
    constexpr int kLds = TileCore<D, true>::kLds;
    static DeviceOnce attr_set;
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (!attr_set.is_done(dev)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(&baps_attn_window_tile_kernel<D, NW>),
                                hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
        if (e != hipSuccess) return e;
        attr_set.mark(dev);
    }
    const long long flat = (long long)p.Sq * (p.Hq / p.Hkv), tiles = (flat + 32 * NW - 1) / (32 * NW);
    hipLaunchKernelGGL((baps_attn_window_tile_kernel<D, NW>), dim3((unsigned)(tiles * p.nsplit * p.Hkv * p.B)), dim3(64 * NW),
                       kLds, st, p);
    e = hipGetLastError();
    return e != hipSuccess || p.nsplit == 1 ? e : launch_window_combine(p, D, st);
}

}  // namespace

hipError_t launch_attention_window_tile(const AttnParams& p, int D, int rows, hipStream_t st)
{
    if (D == 64) return launch_rows<64, 4>(p, st);
    return rows == 128 ? launch_rows<128, 4>(p, st) : launch_rows<128, 8>(p, st);
}

}  // namespace baps
