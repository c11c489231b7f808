// The inner loop of the attention kernels in the Default setup (eq. (2) with
// every softmax operation in fp32) for 32 query rows per wave: half blocks of 32
// keys whose products and exponentials are interleaved by hand.
//
// S^T = K Q^T and O^T += V^T P^T run on v_mfma_f32_32x32x16_bf16; a lane holds one
// row's 16 scores of 32 keys, which are its operand of P V as they stand.
//
// What bounds it: the instructions of a wave.  Per 64 keys and wave, 32 MFMAs
// take 1024 cycles of the SIMD, the exponentials with their exponent, sum and
// packing 740, the maxima 160; two waves share a SIMD.  So the Q^T of the next 32
// keys, the P V of the current ones and the exponentials between them are
// written out in one order (fused), and what depends on one another stands
// apart: a score's exponent, exponential and sum each one MFMA further on, every
// operand read from LDS four MFMAs ahead, the P V of the upper 16 keys in the
// next 32 keys' turn.
#pragma once
#include "common.hpp"

namespace baps {

typedef __bf16 bf16x2 __attribute__((__vector_size__(2 * sizeof(__bf16))));
typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}

// the larger of the values of lanes l and l ^ 32
__device__ __forceinline__ float max_halves(float x)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(hif8::u2f(r[0]), hif8::u2f(r[1]));
}

constexpr int kBlk = 64;            // keys of a block

// Blocks lie in LDS as four half blocks of K, [32 keys][D] (half 2 j of block j in
// slot 2 j % 4), and behind them three blocks of V, rows' 16-byte chunks
// XOR-swizzled: what a step reads, and the next one's on their way.  (Two steps
// ahead, with six and four, measured the same.)
//   TR = false: V as [D][64 keys]; K's rows are taken in the order that gives a
//     lane 8 consecutive keys per 16 (row 8a + 4h + b is key 16 (a/2) + 8h +
//     4 (a%2) + b), so V's operand is one 16-byte read.
//   TR = true: V as it is in memory, [64 keys][D], through the transposing reads;
//     K's rows in their own order.
template <int D, bool TR>
struct TileCore {
    static constexpr int kDK = D / 16, kDT = D / 32;
    static constexpr int kKB = kBlk * D * 2, kHalf = kKB / 2, kVBase = 4 * kHalf, kLds = kVBase + 3 * kKB;

    char* lds;
    float scale;                    // of the scores, in log2 units
    u32x4 qop[kDK];                 // Q^T: row's elements 16 k + 8 (lane / 32) ..
    f32x16 oacc[kDT];
    float m, l, l2, nref;           // reference (log2 units), the two halves of the sum, -m (0 for none)
    u32x4 late;                     // P of the upper 16 of the last 32 keys, and where their V is
    uint32_t late_at;
    uint32_t koff[kDK], voff[TR ? kDT : kBlk / 16];

    __device__ __forceinline__ void init(char* lds_, int lane, float scale_)
    {
        const float ninf = -__builtin_huge_valf();
        const int j32 = lane & 31, half = lane >> 5;
        lds = lds_;
        scale = scale_;
        m = ninf;
        l = l2 = nref = 0.0f;
#pragma unroll
        for (int t = 0; t < kDT; ++t) oacc[t] = f32x16{};
        const int ka = j32 >> 3, kh = (j32 >> 2) & 1;
        const int krow = TR ? j32 : 16 * (ka >> 1) + 8 * kh + 4 * (ka & 1) + (j32 & 3);
        const int kx = D == 128 ? (krow & 15) : ((krow >> 1) & 7);
#pragma unroll
        for (int k = 0; k < kDK; ++k) koff[k] = krow * 2 * D + 16 * ((2 * k + half) ^ kx);
        if constexpr (TR) {
            // transposing reads: lane l of 16 points at row 4 half + (l%16)/4 (+ 8
            // for the second read) and at 4 values of d
            const int s16 = lane & 15, row0 = 4 * half + s16 / 4;
            const int vx = D == 128 ? 2 * (row0 & 3) : 2 * ((row0 >> 1) & 1);
#pragma unroll
            for (int t = 0; t < kDT; ++t) {
                const int d = 32 * t + 16 * ((lane >> 4) & 1) + 4 * (s16 & 3);
                voff[t] = row0 * 2 * D + 16 * ((d >> 3) ^ vx) + 2 * (d & 7);
            }
        } else {
            const int vx = (j32 >> 1) & 7;                      // (the same for row j32 + 32 t)
#pragma unroll
            for (int c = 0; c < kBlk / 16; ++c) voff[c] = j32 * 2 * kBlk + 16 * ((2 * c + half) ^ vx);
        }
        late = u32x4{0, 0, 0, 0};
        late_at = v_at(kVBase, 0);
    }

    // the key of score register r, less 8 (TR: 4) times the lane's half
    static constexpr int key_of(int r) { return TR ? 8 * (r >> 2) + (r & 3) : 16 * (r >> 3) + (r & 7); }
    static constexpr int kKeyHalf = TR ? 4 : 8;

    __device__ __forceinline__ u32x4 k_read(int k, int slot) const
    {
        return *reinterpret_cast<const u32x4*>(lds + koff[k] + slot * kHalf);
    }
    // the 16 keys ch of the block at byte offset buf
    __device__ __forceinline__ uint32_t v_at(uint32_t buf, int ch) const
    {
        if constexpr (TR) return buf + ch * 16 * 2 * D;
        else return buf + voff[ch];
    }
    __device__ __forceinline__ u32x4 v_read(uint32_t at, int t) const
    {
        if constexpr (TR) {
            typedef __attribute__((address_space(3))) s16x4* ptr;
            const char* p = lds + (at + voff[t]);
            const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(p)));
            const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(p + 8 * 2 * D)));
            return u32x4{a[0], a[1], b[0], b[1]};
        } else {
            return *reinterpret_cast<const u32x4*>(lds + at + 32 * t * 2 * kBlk);
        }
    }

    // the first 32 keys' scores
    __device__ __forceinline__ void first(f32x16& sc, int slot)
    {
#pragma unroll
        for (int k = 0; k < kDK; ++k)
            sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(k_read(k, slot)), as_bf16x8(qop[k]), k ? sc : f32x16{}, 0, 0, 0);
    }

    // the late P V
    __device__ __forceinline__ void finish()
    {
#pragma unroll
        for (int t = 0; t < kDT; ++t)
            oacc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(v_read(late_at, t)), as_bf16x8(late), oacc[t], 0, 0, 0);
        late = u32x4{0, 0, 0, 0};
    }

    // The reference that the P of masked scores are formed against.  It is the
    // running maximum only up to a factor of 2^8: it moves when a row's maximum
    // passes it by more, so that the output is rarely rescaled (P stays within 2^8
    // of 1, in floating point at the same relative precision, and the sums in
    // fp32).  FIRST: of the first 32 keys, with nothing summed yet.
    template <bool FIRST>
    __device__ __forceinline__ void settle(const f32x16& sc)
    {
        const float ninf = -__builtin_huge_valf();
        float mx = ninf;
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[r]);
        mx = max_halves(mx) * scale;
        if (__any(mx > m + 8.0f)) {                             // (m = -inf: any finite maximum)
            const float m_new = fmaxf(m, mx);
            const float fac = m == ninf ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
            if constexpr (!FIRST) {
                finish();
#pragma unroll
                for (int t = 0; t < kDT; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r) oacc[t][r] *= fac;
                l *= fac;
                l2 *= fac;
            }
            m = m_new;
            nref = m == ninf ? 0.0f : -m;
        }
    }

    // Q^T of the next 32 keys (slot) and P V of the current ones (half `up` of the
    // block of V at buf) in turn, one MFMA each: first the late 16 keys of the 32
    // before, then the current lower 16.  The current scores turn into P between
    // them.  (The order is written out: left to the compiler, the reads come one
    // MFMA ahead and the exponentials in a bunch.)
    __device__ __forceinline__ void fused(const f32x16& cur, f32x16& nxt, int slot, uint32_t buf, int up)
    {
        constexpr int kN = 2 * kDK, kAhead = 4, kPerSlot = 16 / kN, kLead = 4;
        static_assert(kDK == 2 * kDT && 16 % kN == 0, "as many MFMAs of Q^T as of P V, one score or more beside each");
        const uint32_t vlow = v_at(buf, 2 * up);
        auto operand = [&](int i) {
            if (i & 1) return k_read(i >> 1, slot);
            const int n = i >> 1;                               // P V: n < kDT late, then the current lower 16 keys
            return n < kDT ? v_read(late_at, n) : v_read(vlow, n - kDT);
        };
        u32x4 fr[kAhead], pop[2];
        float x[16];
        auto stage = [&](int r, int s) {
            if (r < 0 || r >= 16) return;
            if (s == 0) x[r] = __builtin_fmaf(cur[r], scale, nref);
            if (s == 1) x[r] = __builtin_amdgcn_exp2f(x[r]);
            if (s == 2) {
                if (r & 1) l2 += x[r]; else l += x[r];
                if (r & 1) pop[r >> 3][(r & 7) >> 1] = pack_bf16(x[r - 1], x[r]);
            }
        };
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) fr[i] = operand(i);
#pragma unroll
        for (int r = 0; r < kLead; ++r) stage(r, 0);
#pragma unroll
        for (int r = 0; r < kLead - 2; ++r) stage(r, 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const bf16x8 a = as_bf16x8(fr[i % kAhead]);
            const int n = i >> 1;
            if (i & 1) nxt = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, as_bf16x8(qop[n]), n ? nxt : f32x16{}, 0, 0, 0);
            else oacc[n % kDT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, as_bf16x8(n < kDT ? late : pop[0]), oacc[n % kDT], 0, 0, 0);
            if (i + kAhead < kN) fr[i % kAhead] = operand(i + kAhead);
#pragma unroll
            for (int e = 0; e < kPerSlot; ++e) {
                const int r = kPerSlot * i + e;
                stage(r + kLead, 0);
                stage(r + kLead - 2, 1);
                stage(r + kLead - 4, 2);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        late = pop[1];
        late_at = v_at(buf, 2 * up + 1);
        // (formed here, not where it is read)
        asm volatile("" : "+v"(late[0]), "+v"(late[1]), "+v"(late[2]), "+v"(late[3]));
    }

    // the buffer of the next block of V
    __device__ __forceinline__ static uint32_t next_v(uint32_t buf)
    {
        return buf == (uint32_t)(kVBase + 2 * kKB) ? (uint32_t)kVBase : buf + kKB;
    }

    // the row's sum over both halves of the lanes
    __device__ __forceinline__ float total() const
    {
        const float s = l + l2;
        return s + __shfl_xor(s, 32, 64);
    }
    // register r of tile t of O^T is element 32 t + 8 (r/4) + 4 (lane / 32) + r%4
    __device__ __forceinline__ f32x4 out4(int t, int q, float f) const
    {
        return f32x4{oacc[t][4 * q] * f, oacc[t][4 * q + 1] * f, oacc[t][4 * q + 2] * f, oacc[t][4 * q + 3] * f};
    }
};

}  // namespace baps
