// Shared device-side helpers and launch descriptors of the BAPS HIP library.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "hif8.hpp"

namespace baps {

// Host-side set-up done once per device and kernel (a launch attribute, an
// occupancy query): one bit per device ordinal below 64, set once the step
// succeeded there.  Concurrent first calls may both run the step, which is
// idempotent.  Ordinals from 64 up run it on every call.
struct DeviceOnce {
    std::atomic<unsigned long long> done{0};
    bool is_done(int dev) const
    {
        return dev >= 0 && dev < 64 && (done.load(std::memory_order_acquire) >> dev & 1ull);
    }
    void mark(int dev)
    {
        if (dev >= 0 && dev < 64) done.fetch_or(1ull << dev, std::memory_order_release);
    }
};

// Compute units of the current device, read once per device ordinal below 64.
inline hipError_t cu_count(int* ncu)
{
    static std::atomic<int> count[64] = {};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const bool kept = dev >= 0 && dev < 64;
    *ncu = kept ? count[dev].load(std::memory_order_relaxed) : 0;
    if (*ncu) return hipSuccess;
    e = hipDeviceGetAttribute(ncu, hipDeviceAttributeMultiprocessorCount, dev);
    if (e == hipSuccess && kept) count[dev].store(*ncu, std::memory_order_relaxed);
    return e;
}

typedef __bf16 bf16x8 __attribute__((__vector_size__(8 * sizeof(__bf16))));
typedef float f32x16 __attribute__((__vector_size__(16 * sizeof(float))));
typedef float f32x4 __attribute__((__vector_size__(4 * sizeof(float))));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Entries of the score table, indexed by bits 31..19 of an fp32 value T:
// P = HiF8(2^HiF8(T)) as fp32 bits in bits 31..8, and the HiF8 code of P in
// bits 7..0 (every HiF8 value has at most 3 mantissa bits, so bits 19..0 of
// its fp32 pattern are zero).  The upper 16 bits are P in bf16, exactly.
constexpr int kTabEntries = 8192;
constexpr int kTabShift = 19;

// Compact code table of the fused attention kernels, for thresholds lambda
// <= kCodeMaxLambda.  Indexed like the score table (bits 31..19 of T) but
// clamped to [kCodeLo, kCodeHi]: every T <= lambda lands on an entry with the
// same P, since P = 1 for |T| < 2^-5 (either sign; the clamp sends positive T
// below 2^-5 to the entry of 2^-5) and P = 0 for T <= -32 (the clamp sends
// -inf and every T <= -32 to the entry of -32).  An entry is the byte
// c = ((e + 23) << 3) | m of P = 2^e (1 + m/8) (c = 0 for P = 0), chosen so
// that c << 4 is the bf16 pattern of P * 2^-kCodeBiasLog2, exactly: e runs
// over [-22, kCodeMaxLambda] and HiF8 keeps at most 3 mantissa bits.  In
// practice the hit entries sit in a few dozen LDS dwords: the gathers are
// nearly free of bank conflicts.  The prefill kernel expands the table in LDS
// to all 8192 indices (entry kCodeLo below, kCodeHi above the range), which
// takes the clamp off every lookup.
constexpr int kCodeLo = 0x7A0;           // T = +2^-5
constexpr int kCodeHi = 0x1840;          // T = -32
constexpr int kCodeEntries = kCodeHi - kCodeLo + 1;
constexpr int kCodeTableBytes = (kCodeEntries + 1023) / 1024 * 1024;   // device copy, zero-padded to whole KiB
constexpr int kCodeBiasLog2 = 104;
constexpr int kCodeMaxLambda = 8;

// max(0, ceil(HiF8(x))) (ties away) for x below 8.75, branch-free: below
// 2^-23 the cast gives 0 or less; from 2^-23 up to 16 it keeps at most 3
// mantissa bits, so with h half the spacing of x's binade (2^(e-4) in
// [2^e, 2^(e+1)) for e >= 0, below the spacing for e < 0) the cast exceeds an
// integer k exactly when x >= k + h (ties go away from zero), and
// ceil(HiF8(x)) = floor(x - h) + 1; x - h is exact (h is at least one unit in
// the last place of x).  Alg. 1's increment of the integer maximum when a
// block does not restart (T <= lambda <= 8).
__device__ __forceinline__ float hif8_ceil_below9(float x)
{
    const float h = hif8::u2f((hif8::f2u(x) & 0x7f800000u) - (4u << 23));
    const float r = floorf(x - h) + 1.0f;
    return x >= 0x1p-23f ? r : 0.0f;
}

// 2^k for an integer-valued k <= 0 (0 below the fp32 range)
__device__ __forceinline__ float exp2_nonpos_int(float k)
{
    return ldexpf(1.0f, (int)__builtin_fmaxf(k, -200.0f));
}

// Softmax setups of the fused attention kernels: the proposed workflow
// (Alg. 1, "E2E HiF8") and two setups of eq. (2) with a real-valued running
// maximum, "Default" (fp32 exp2) and "Exp2 HiF8" (the exp2 evaluated on 8-bit
// input and rounded to 8 bits), for comparison on the same tiling.
constexpr int kModeE2E = 0;
constexpr int kModeDefault = 1;
constexpr int kModeExp2 = 2;
// The kernels' MODE of a windowed call: the setup with this bit set
constexpr int kModeWindow = 8;

struct AttnParams {
    const uint16_t* q;          // [B, Hq, Sq, D] bf16
    const uint16_t* k;          // [B, Hkv, Sk, D] bf16
    const uint16_t* v;          // [B, Hkv, Sk, D] bf16
    float* o;                   // [B, Hq, Sq, D]
    float* lse;                 // [B, Hq, Sq] or null
    const uint32_t* tab;        // score table (device)
    const uint8_t* ctab;        // compact code table (device), kCodeTableBytes bytes (entries, then zeros)
    const uint8_t* ctabx;       // the compact code table expanded to all kTabEntries indices (device)
    float dec_x0;               // the least fp32 T with ceil(HiF8(T)) > lambda (ties away): Alg. 1's
                                // restart test is T >= dec_x0
    unsigned long long* counters;  // [B*Hq][2] restarted / visited B1 tile-blocks, or null
    unsigned long long* tile_counts;  // [B*Hq][ceil(Sq/R)][2] the same per tile, or null
    int B, Hq, Hkv, Sq, Sk;
    int causal, lambda, n_b0;
    int mode;                   // kModeE2E, kModeDefault or kModeExp2
    int restart_rows;           // R: query positions of one head sharing the restart decision
    int b0_last;                // B0 also holds each row's last visible key block
    int qk_f8;                  // q and k hold FP8 E4M3 codes (c already holds the scales)
    float c;                    // log2(e)/sqrt(D) as fp32 (or the caller's override)
    int out_bf16;               // o holds bf16 (round to nearest even of the fp32 result)
    int tie_even;               // the 8-bit cast of T rounds ties to even (kernels built with TIE)
    const uint8_t* ctab_even;   // compact code table for exact ties under ties-to-even (device)
    const uint8_t* ctabx_even;  // the same expanded to all kTabEntries indices (device)
    // Score dump (kernels built with DUMP only): a query row whose
    // dump_slot[(b*Hq + h)*Sq + r] is s >= 0 writes its raw dot products q.k
    // to dump_acc[s*Sk + key] for every key it sees, and its reference (Alg.
    // 1's m~; the running maximum in the eq. (2) setups) after every key block
    // j it sees to dump_ref[s*dump_nblk + j]
    const int* dump_slot;
    float* dump_acc;
    float* dump_ref;
    int dump_nblk;
    // Windowed calls (kernels built with kModeWindow): the row at position t
    // sees key c <= t when c > t - window or c < sinks
    int window, sinks;
    // and in the Default setup with few rows the keys may be split over nsplit
    // workgroups: [nsplit][B*Hq*Sq] unnormalised sums and (maximum, sum) pairs
    int nsplit;
    float* part;                // [..][D]
    float* ml;                  // [..][2]
};

// Key blocks of KB keys that the rows at positions t_lo .. t_hi reach: the
// sinks' blocks first, then the window's, as one list of n blocks.  window 0:
// every key up to the row.
struct KeyBlocks {
    int nsink, wstart, n, lo;       // lo: the first key of the window of the lowest row
    __device__ __forceinline__ int block(int j) const { return j < nsink ? j : wstart + (j - nsink); }
};

template <int KB>
__device__ __forceinline__ KeyBlocks key_blocks(int t_lo, int t_hi, int window, int sinks)
{
    KeyBlocks r;
    r.lo = window > 0 ? max(0, t_lo - window + 1) : 0;
    const int ns = min(min(sinks, r.lo), t_hi + 1);             // sink keys in front of the window
    r.wstart = r.lo / KB;
    r.nsink = ns > 0 ? min((ns + KB - 1) / KB, r.wstart) : 0;
    r.n = t_hi < 0 ? 0 : r.nsink + (t_hi / KB - r.wstart + 1);
    return r;
}

// Zeros over the rows of an LDS block of V (n keys from key0 on, ROW_BYTES each)
// that are no sinks and lie in front of lo: nobody's window holds them, their
// weights are zero, and they may be anything, NaN included.  By `threads`
// threads, of which this is number t.
template <int ROW_BYTES>
__device__ __forceinline__ void zero_hidden_v(char* v, int key0, int n, int lo, int sinks, int t, int threads)
{
    const int r1 = min(lo - key0, n);
    for (int i = max(sinks - key0, 0) * (ROW_BYTES / 16) + t; i < r1 * (ROW_BYTES / 16); i += threads)
        *reinterpret_cast<u32x4*>(v + 16 * i) = u32x4{0, 0, 0, 0};
}

struct SoftmaxBlockParams {
    const float* s;
    long long rows, cols, ld;
    int block, lambda, n_b0;
    uint8_t* codes;
    int32_t* ref_shift;
    float* m_final;
    float* d_final;
    uint8_t* restarted;
    const uint32_t* tab;
};

// The split-key path of the few-rows kernels (decode with few (batch, KV
// head) streams and many keys).  Alg. 1's state after block j depends on the
// key blocks only through their row maxima, so the path runs in passes over
// a caller-provided workspace: the raw dot products and block maxima of every
// key split in parallel; then, per split in parallel, a per-row scan of Alg.
// 1's restart rule and integer maximum up to the split and P V at the
// references of that scan; last, per row, an exact power-of-two combine.
// The result is the sequential one up to the order of fp32 additions.
struct SplitParams {
    AttnParams a;               // the attention call (mode kModeE2E, lambda <= kCodeMaxLambda)
    float* acc;                 // [B*Hkv][flat][nblk*BLK] raw dot products q.k (-inf when masked)
    float* bmax;                // [B*Hkv][flat][bstride] raw row maximum of every key block
    float* part;                // [nsplit][B*Hkv][flat][D + 4] X, dX and the reference they are relative to
    int nblk, bstride;          // key blocks, and the block-maximum row stride (a multiple of 256)
    int nsplit, bps;            // splits, blocks per split (at most kSplitMaxBps)
};

constexpr int kSplitMaxBps = 32;  // key blocks per split of the split-key path

// exact 2^k for an integer-valued float k (0 below the fp32 range)
__device__ __forceinline__ float exp2_int(float k)
{
    if (k < -160.0f) return 0.0f;
    return ldexpf(1.0f, (int)k);
}

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    return v;
}

// Wave-uniform maximum with DPP row ops (quad permutes and mirrors inside
// each row of 16 lanes, then row broadcasts): no LDS round trips.
__device__ __forceinline__ float dpp_max_step(float v, int ctrl, int row_mask)
{
    const int o = __builtin_bit_cast(int, v);
    switch (ctrl) {   // the DPP control must be a compile-time constant
    case 0xB1: return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(o, o, 0xB1, 0xF, 0xF, false)));
    case 0x4E: return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(o, o, 0x4E, 0xF, 0xF, false)));
    case 0x141: return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(o, o, 0x141, 0xF, 0xF, false)));
    case 0x140: return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(o, o, 0x140, 0xF, 0xF, false)));
    case 0x142: return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(o, o, 0x142, 0xA, 0xF, false)));
    default: return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(o, o, 0x143, 0xC, 0xF, false)));
    }
}

__device__ __forceinline__ float wave_max_uniform(float v)
{
    v = dpp_max_step(v, 0xB1, 0xF);     // lane ^ 1
    v = dpp_max_step(v, 0x4E, 0xF);     // lane ^ 2
    v = dpp_max_step(v, 0x141, 0xF);    // mirror within 8
    v = dpp_max_step(v, 0x140, 0xF);    // mirror within 16
    v = dpp_max_step(v, 0x142, 0xA);    // row 0 -> 1, row 2 -> 3
    v = dpp_max_step(v, 0x143, 0xC);    // row 1 -> 2 and 3
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}

// Lanes in groups of L (16, 32 or 64): the maximum of v over the lower lanes of
// the group, -inf for its first lane
template <int L>
__device__ __forceinline__ float prefix_max_before(float v)
{
    const float ninf = -__builtin_huge_valf();
    const int ni = __builtin_bit_cast(int, ninf);
#define BAPS_STEP(CTRL, ROWS)                                                                                     \
    v = __builtin_fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(ni, __builtin_bit_cast(int, v),  \
                                                                                 CTRL, ROWS, 0xF, false)))
    BAPS_STEP(0x111, 0xF);                        // row_shr 1, 2, 4, 8: inclusive maxima within 16 lanes
    BAPS_STEP(0x112, 0xF);
    BAPS_STEP(0x114, 0xF);
    BAPS_STEP(0x118, 0xF);
    if constexpr (L >= 32) BAPS_STEP(0x142, 0xA);   // lane 15 of rows 0 and 2 to rows 1 and 3
    if constexpr (L == 64) BAPS_STEP(0x143, 0xC);   // lane 31 to rows 2 and 3
#undef BAPS_STEP
    const float before = __shfl_up(v, 1, 64);
    return (threadIdx.x & (L - 1)) == 0 ? ninf : before;
}

// Host launchers (one per kernel family); return a hipError_t.
hipError_t launch_hif8_encode(const float* x, uint8_t* codes, long long n, bool saturate, bool even, hipStream_t st);
hipError_t launch_hif8_decode(const uint8_t* codes, float* x, long long n, hipStream_t st);
hipError_t launch_softmax_block(const SoftmaxBlockParams& p, hipStream_t st);
hipError_t launch_attention(const AttnParams& p, int D, int block, hipStream_t st);
hipError_t launch_attention_dump(const AttnParams& p, int D, int block, hipStream_t st);
hipError_t launch_attention_decode(const AttnParams& p, int D, int block, hipStream_t st);
hipError_t launch_attention_split(const SplitParams& sp, int D, int block, hipStream_t st);
hipError_t launch_attention_window(const AttnParams& p, int D, int block, hipStream_t st);
hipError_t launch_attention_window_few(const AttnParams& p, int D, int block, hipStream_t st);
hipError_t launch_attention_window_tile(const AttnParams& p, int D, int rows, hipStream_t st);
hipError_t launch_window_combine(const AttnParams& p, int D, hipStream_t st);

// Which kernel a windowed Default call with many rows takes.  Where 128-row items
// all run at once, one to a CU, the latency of a step sets the time, and the kernel
// of attn_fwd.hpp with 128-key blocks wins, whose keys are split over two waves (GQA
// 32/8, D = 128: 512 positions, window 256, 13.9 us against the tile kernel's 16.6;
// 900, 1700: 41 against 50; 16 heads of 600 at D = 64, 300: 13.9 against 15.5).  With
// items for a third of the CUs only and more than 1536 keys, the tile kernel's
// workgroups split the keys (100 positions, window 4096: 58 -> 29 us, 100 whole; with
// items for half of the CUs, 16 heads of 1000 at D = 64, 2000, it would be 27 -> 30,
// the parts' join being most of it).  With more items the products bind, and the
// tile kernel wins (16384 positions, window 4096: 1020 -> 973 us; D = 64, 16 heads
// of 2300, 4000: 89 -> 84).  At D = 128, two workgroups of 128 rows on a CU fill each
// other's starts and ends, one of 256 rows loads K and V half as often: up to 2048
// keys the former (16384 positions, window 256: 189 -> 170 us; 4 x 32 heads of 2000:
// 180 -> 174), then the latter (16384, 4096: 974 against 995; 4096, 4096: 147
// against 154).
struct WindowForm {
    int rows;                       // of a workgroup: 64 or 128 (two waves on the same rows) ..
    bool tile;                      // .. or, of the tile kernel, 128 or 256
    long long keys;                 // tile: that a workgroup's rows reach, at most, where they are to be split; else 0
};

inline WindowForm window_form(int D, long long flat, int group, long long heads, long long Sk, long long window,
                              long long sinks, int ncu)
{
    const long long n64 = (flat + 63) / 64 * heads, n128 = (flat + 127) / 128 * heads;
    const long long reach = window + sinks + 128 / group + 1, keys = reach < Sk ? reach : Sk;
    if (3 * n128 <= ncu && keys > 1536) return {128, true, keys};
    if (n128 <= ncu) return {D == 64 || n64 <= ncu ? 64 : 128, false, 0};
    return {D == 64 || keys <= 2048 ? 128 : 256, true, 0};
}

// rows per key/value head up to which a call takes the few-rows kernel
constexpr long long kFewFlatRows = 64;

}  // namespace baps
