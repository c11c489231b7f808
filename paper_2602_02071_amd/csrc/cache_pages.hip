// The pages of the cache: fork (share, copy, take and free pages as sequences
// go on from others) and compact (close the holes of a pool).
//
// A page's state is its reference count alone; free pages are those with count
// zero and are taken lowest first, so a result depends on the counts and
// tables only and is the same on every run (counts move by integer atomics,
// whose order does not show).  The copies move whole pages of all layers,
// 16 bytes per lane, and are bound by memory (3000 pages of 64 tokens, four
// layers, 45 % of them holes: 778 MB in 155 us, the rate of a copy); the
// bookkeeping is a few thousand integers and bound by latency.
#include "cache.hpp"

namespace baps {

namespace {

constexpr int kScan = 1024;         // threads of the kernels that rank free pages

__device__ __forceinline__ bool valid_page(int page, int num_pages) { return (unsigned)page < (unsigned)num_pages; }

// Exclusive prefix sum of v over the workgroup's kScan threads; *total: the
// sum.  tmp: kScan / 64 words of LDS.
__device__ __forceinline__ int block_scan(int v, int* tmp, int* total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
    }
    __syncthreads();                                            // (tmp of the scan before is read)
    if (lane == 63) tmp[wave] = x;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kScan / 64; ++w) {
        const int t = tmp[w];
        before += w < wave ? t : 0;
        all += t;
    }
    *total = all;
    return before + x - v;
}

// ---------------------------------------------------------------- fork
// What child i takes over from its parent and what it needs.
struct Child {
    int len, src, taken, fresh, over;
};

template <class Refs>
__device__ __forceinline__ Child plan_child(const CacheForkParams& p, int i, bool first, const Refs& refs)
{
    const int par = p.parent[i];
    int len = 0, full = 0, copied = 0, src = -1;
    if (valid_page(par, p.B_in)) {
        len = (int)min((long long)max(p.lens_in[par], 0), (long long)p.width * p.page);
        full = (len + p.page - 1) / p.page;
        if (len % p.page) {
            // a partly filled last page is written by the next append, so only
            // one sequence may hold it
            const int tail = p.table_in[(long long)par * p.width + full - 1];
            if (valid_page(tail, p.num_pages) && !(first && refs[tail] == 1)) {
                src = tail;
                copied = 1;
            }
        }
    }
    const long long grow = p.grow ? max(p.grow[i], 0) : 0;
    const long long more = (len + grow + p.page - 1) / p.page;        // pages in all
    // (pages past the table's width are held so low that their sum over the
    // children stays below 2^30)
    return Child{len, src, full - copied, (int)min(more, (long long)p.width) - full + copied,
                 (int)min(max(more - p.width, 0LL), (1LL << 30) / p.B_out)};
}

// A page that this call copies from is not taken by it, even if nothing holds it
// any more: between counting and ranking its count reads kRead.
constexpr int kRead = -0x7fffffff - 1;

// The child that the rank-th fresh page goes to: first[c] <= rank < first[c + 1]
__device__ __forceinline__ int child_of(const int* first, int n, int rank)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= rank) lo = mid; else hi = mid;
    }
    return lo;
}

// The whole bookkeeping in one workgroup, the references and the children's
// numbers in LDS: one launch in place of three (8 children of 8 sequences, with
// the copies, 21.1 -> 18.8 us; at 11600 table entries, 192 of 160 sequences, both
// take 24.5, and more entries are more than one workgroup should walk).
// kSmallWords: what LDS holds.
constexpr int kSmallWords = 32768, kSmallEntries = 8192;

bool fork_is_small(const CacheForkParams& p)
{
    return (long long)p.num_pages + p.B_in + 5LL * p.B_out + 1 <= kSmallWords &&
           ((long long)p.B_in + p.B_out) * p.width <= kSmallEntries;
}

__global__ __launch_bounds__(kScan) void baps_cache_fork_small_kernel(CacheForkParams p)
{
    extern __shared__ int words[];
    __shared__ int tmp[kScan / 64];
    int* refs = words;                                          // [num_pages]
    int* first = refs + p.num_pages;                            // [B_in] a parent's first child
    int* src = first + p.B_in;                                  // [B_out] each
    int* dst = src + p.B_out;
    int* taken = dst + p.B_out;
    int* par = taken + p.B_out;
    int* fresh = par + p.B_out;                                 // [B_out + 1]
    const int tid = threadIdx.x;
    for (int i = tid; i < p.num_pages; i += kScan) refs[i] = p.refs_in[i];
    for (int i = tid; i < p.B_in; i += kScan) first[i] = 0x7fffffff;
    __syncthreads();
    for (int i = tid; i < p.B_out; i += kScan) {
        par[i] = p.parent[i];
        if (valid_page(par[i], p.B_in)) atomicMin(first + par[i], i);
    }
    __syncthreads();
    int over = 0, total;
    for (int i = tid; i < p.B_out; i += kScan) {
        const Child c = plan_child(p, i, valid_page(par[i], p.B_in) && first[par[i]] == i, refs);
        p.lens_out[i] = c.len;
        src[i] = c.src;
        dst[i] = -1;
        taken[i] = c.taken;
        fresh[i] = c.fresh;
        over += c.over;
    }
    __syncthreads();
    // (kAtOnce entries of a thread are loaded before the first is used)
    constexpr int kAtOnce = 4;
    for (int i0 = tid; i0 < p.B_in * p.width; i0 += kAtOnce * kScan) {
        int page[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) page[u] = i0 + u * kScan < p.B_in * p.width ? p.table_in[i0 + u * kScan] : -1;
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
            if (valid_page(page[u], p.num_pages)) atomicSub(refs + page[u], 1);
    }
    for (int i0 = tid; i0 < p.B_out * p.width; i0 += kAtOnce * kScan) {
        int page[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int i = i0 + u * kScan, r = min(i / p.width, p.B_out - 1), c = i - r * p.width;
            page[u] = c < taken[r] ? p.table_in[par[r] * p.width + c] : -1;
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int i = i0 + u * kScan;
            if (i >= p.B_out * p.width) break;
            const bool ok = valid_page(page[u], p.num_pages);
            if (ok) atomicAdd(refs + page[u], 1);
            p.table_out[i] = ok ? page[u] : -1;
        }
    }
    // fresh[i] becomes the rank of child i's first fresh page
    int want = 0;
    for (int i0 = 0; i0 < p.B_out; i0 += kScan) {
        const int i = i0 + tid, v = i < p.B_out ? fresh[i] : 0;
        const int at = block_scan(v, tmp, &total);
        if (i < p.B_out) fresh[i] = want + at;
        want += total;
    }
    __syncthreads();                                            // references and table rows are whole
    for (int i = tid; i < p.B_out; i += kScan)
        if (src[i] >= 0) atomicCAS(refs + src[i], 0, kRead);
    __syncthreads();
    // every thread ranks the free pages of a run of its own
    const int run = (p.num_pages + kScan - 1) / kScan, p0 = min(tid * run, p.num_pages), p1 = min(p0 + run, p.num_pages);
    int n = 0, found;
    for (int i = p0; i < p1; ++i) n += refs[i] == 0;
    int rank = block_scan(n, tmp, &found);
    for (int i = p0; i < p1 && rank < want; ++i) {
        if (refs[i] != 0) continue;
        const int c = child_of(fresh, p.B_out, rank), k = rank - fresh[c];
        p.table_out[c * p.width + taken[c] + k] = i;
        refs[i] = 1;
        if (k == 0 && src[c] >= 0) dst[c] = i;
        ++rank;
    }
    block_scan(over, tmp, &total);                              // (its barriers publish refs and dst)
    if (tid == 0) p.missing[0] = want - min(found, want) + total;
    for (int i = tid; i < p.num_pages; i += kScan) p.refs_out[i] = refs[i] == kRead ? 0 : refs[i];
    for (int i = tid; i < p.B_out; i += kScan) {
        p.src[i] = src[i];
        p.dst[i] = dst[i];
    }
}

__global__ __launch_bounds__(256) void baps_cache_fork_plan_kernel(CacheForkParams p)
{
    __shared__ int twin;
    const int i = blockIdx.x;
    if (i < p.B_out) {
        if (threadIdx.x == 0) twin = 0;
        __syncthreads();
        const int par = p.parent[i];
        bool t = false;
        for (int k = threadIdx.x; k < i; k += 256) t |= p.parent[k] == par;
        if (t) twin = 1;
        __syncthreads();
        if (threadIdx.x == 0) {
            const Child c = plan_child(p, i, !twin, p.refs_in);
            p.lens_out[i] = c.len;
            p.src[i] = c.src;
            p.dst[i] = -1;
            p.taken[i] = c.taken;
            p.fresh[i] = c.fresh;
            p.over[i] = c.over;
        }
    }
    if (p.refs_out != p.refs_in)
        for (long long k = (long long)blockIdx.x * 256 + threadIdx.x; k < p.num_pages; k += (long long)gridDim.x * 256)
            p.refs_out[k] = p.refs_in[k];
}

__global__ __launch_bounds__(256) void baps_cache_fork_refs_kernel(CacheForkParams p)
{
    const int r = blockIdx.x;
    if (r < p.B_out) {
        const int taken = p.taken[r];
        const int* from = p.table_in + (long long)(taken > 0 ? p.parent[r] : 0) * p.width;
        int* row = p.table_out + (long long)r * p.width;
        for (int c = threadIdx.x; c < p.width; c += 256) {
            int page = -1;
            if (c < taken) {
                page = from[c];
                if (valid_page(page, p.num_pages)) atomicAdd(p.refs_out + page, 1);
                else page = -1;
            }
            row[c] = page;
        }
    } else {
        const int* row = p.table_in + (long long)(r - p.B_out) * p.width;
        for (int c = threadIdx.x; c < p.width; c += 256) {
            const int page = row[c];
            if (valid_page(page, p.num_pages)) atomicSub(p.refs_out + page, 1);
        }
    }
}

__global__ __launch_bounds__(kScan) void baps_cache_fork_assign_kernel(CacheForkParams p)
{
    __shared__ int tmp[kScan / 64];
    const int tid = threadIdx.x;
    // fresh[i] becomes the rank of child i's first fresh page
    int want = 0, over = 0, total;
    for (int i0 = 0; i0 < p.B_out; i0 += kScan) {
        const int i = i0 + tid;
        const int v = i < p.B_out ? p.fresh[i] : 0;
        over += i < p.B_out ? p.over[i] : 0;
        const int at = block_scan(v, tmp, &total);
        if (i < p.B_out) p.fresh[i] = want + at;
        want += total;
    }
    if (tid == 0) p.fresh[p.B_out] = want;
    for (int i = tid; i < p.B_out; i += kScan)
        if (p.src[i] >= 0) atomicCAS(p.refs_out + p.src[i], 0, kRead);
    __syncthreads();
    int found = 0;
    for (long long p0 = 0; p0 < p.num_pages && found < want; p0 += kScan) {
        const int page = (int)(p0 + tid);
        const bool is_free = page < p.num_pages && p.refs_out[page] == 0;
        const int rank = found + block_scan(is_free ? 1 : 0, tmp, &total);
        found += total;
        if (!is_free || rank >= want) continue;
        const int lo = child_of(p.fresh, p.B_out, rank);
        const int k = rank - p.fresh[lo];
        p.table_out[(long long)lo * p.width + p.taken[lo] + k] = page;
        p.refs_out[page] = 1;
        if (k == 0 && p.src[lo] >= 0) p.dst[lo] = page;
    }
    block_scan(over, tmp, &total);                              // (its barriers end the ranking)
    if (tid == 0) p.missing[0] = want - min(found, want) + total;
    for (int i = tid; i < p.B_out; i += kScan)
        if (p.src[i] >= 0) atomicCAS(p.refs_out + p.src[i], kRead, 0);
}

// ---------------------------------------------------------------- copies
// Page src to page dst of one layer: K, V and their exponents.
__device__ __forceinline__ void copy_page(uint8_t* k, uint8_t* v, uint8_t* ke, uint8_t* ve, int Hkv, long long page_bytes,
                                          long long src, long long dst, int part, int parts)
{
    const long long n = Hkv * page_bytes / 16;                  // 16-byte pieces
    const u32x4* ks = reinterpret_cast<const u32x4*>(k) + src * n;
    const u32x4* vs = reinterpret_cast<const u32x4*>(v) + src * n;
    u32x4* kd = reinterpret_cast<u32x4*>(k) + dst * n;
    u32x4* vd = reinterpret_cast<u32x4*>(v) + dst * n;
    for (long long i = (long long)part * 256 + threadIdx.x; i < n; i += 256LL * parts) {
        const u32x4 a = ks[i], b = vs[i];
        kd[i] = a;
        vd[i] = b;
    }
    if (part == 0)
        for (int i = threadIdx.x; i < Hkv; i += 256) {
            ke[dst * Hkv + i] = ke[src * Hkv + i];
            ve[dst * Hkv + i] = ve[src * Hkv + i];
        }
}

constexpr int kParts = 4;           // workgroups per page and layer

__global__ __launch_bounds__(256) void baps_cache_fork_copy_kernel(CacheForkParams p)
{
    const int i = blockIdx.x, layer = blockIdx.y;
    const int src = p.src[i], dst = p.dst[i];
    if (src < 0 || dst < 0) return;
    const long long bytes = (long long)p.page * p.D, at = (long long)layer * p.num_pages * p.Hkv;
    copy_page(p.k + at * bytes, p.v + at * bytes, p.ke + at, p.ve + at, p.Hkv, bytes, src, dst, blockIdx.z, kParts);
}

// ---------------------------------------------------------------- compact
// The n live pages end up on [0, n): the k-th hole below n takes the k-th live
// page from n up.  Sources lie behind every target, so the moves need no order.
// (Bound by its barriers: 4 us for 512 pages, 7 for 3000; with the references in
// LDS and a run of pages per thread it takes the same.)
__global__ __launch_bounds__(kScan) void baps_cache_compact_plan_kernel(CacheCompactParams p)
{
    __shared__ int tmp[kScan / 64];
    const int tid = threadIdx.x;
    int mine = 0, n;
    for (int i = tid; i < p.num_pages; i += kScan) mine += p.refs_in[i] > 0;
    block_scan(mine, tmp, &n);
    int holes = 0, movers = 0, total;
    for (long long p0 = 0; p0 < p.num_pages; p0 += kScan) {
        const int page = (int)(p0 + tid);
        const bool in = page < p.num_pages;
        const int refs = in ? p.refs_in[page] : 0;
        const bool held = refs > 0;
        const bool hole = in && page < n && !held, mover = in && page >= n && held;
        // (one scan for both: at most kScan of each, 16 bits apart)
        const int at = block_scan((hole ? 1 : 0) + (mover ? 1 << 16 : 0), tmp, &total);
        if (hole) p.to[holes + (at & 0xffff)] = page;
        if (mover) {
            p.from[movers + (at >> 16)] = page;
            p.held[movers + (at >> 16)] = refs;
        }
        if (in) {
            p.remap[page] = held && page < n ? page : -1;
            p.refs_out[page] = page < n ? refs : 0;
        }
        holes += total & 0xffff;
        movers += total >> 16;
    }
    __syncthreads();
    for (int k = tid; k < movers; k += kScan) {
        p.remap[p.from[k]] = p.to[k];
        p.refs_out[p.to[k]] = p.held[k];
    }
    if (tid == 0) {
        p.moves[0] = movers;
        p.live[0] = n;
    }
}

__global__ __launch_bounds__(256) void baps_cache_compact_move_kernel(CacheCompactParams p, int table_groups)
{
    if ((int)blockIdx.x < table_groups) {
        for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < p.entries; i += 256LL * table_groups) {
            const int page = p.table_in[i];
            p.table_out[i] = valid_page(page, p.num_pages) ? p.remap[page] : -1;
        }
        return;
    }
    const long long jobs = (long long)p.moves[0] * p.layers * kParts;
    const long long bytes = (long long)p.page * p.D;
    for (long long j = blockIdx.x - table_groups; j < jobs; j += gridDim.x - table_groups) {
        const int part = (int)(j % kParts);
        const int k = (int)(j / kParts % p.moves[0]);
        const long long at = j / kParts / p.moves[0] * p.num_pages * p.Hkv;
        copy_page(p.k + at * bytes, p.v + at * bytes, p.ke + at, p.ve + at, p.Hkv, bytes, p.from[k], p.to[k], part, kParts);
    }
}

}  // namespace

hipError_t launch_cache_fork(const CacheForkParams& p, hipStream_t st)
{
    hipError_t e;
    if (fork_is_small(p)) {
        static DeviceOnce attr_set;
        int dev = 0;
        if ((e = hipGetDevice(&dev)) != hipSuccess) return e;
        if (!attr_set.is_done(dev)) {
            e = hipFuncSetAttribute(reinterpret_cast<const void*>(&baps_cache_fork_small_kernel),
                                    hipFuncAttributeMaxDynamicSharedMemorySize, 4 * kSmallWords);
            if (e != hipSuccess) return e;
            attr_set.mark(dev);
        }
        const int bytes = 4 * (p.num_pages + p.B_in + 5 * p.B_out + 1);
        hipLaunchKernelGGL(baps_cache_fork_small_kernel, dim3(1), dim3(kScan), bytes, st, p);
    } else {
        const int copies = p.refs_out != p.refs_in ? (p.num_pages + 1023) / 1024 : 0;
        const int g = p.B_out > copies ? p.B_out : (copies > 0 ? copies : 1);
        hipLaunchKernelGGL(baps_cache_fork_plan_kernel, dim3((unsigned)g), dim3(256), 0, st, p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        if (p.B_out + p.B_in > 0) {
            hipLaunchKernelGGL(baps_cache_fork_refs_kernel, dim3((unsigned)(p.B_out + p.B_in)), dim3(256), 0, st, p);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        hipLaunchKernelGGL(baps_cache_fork_assign_kernel, dim3(1), dim3(kScan), 0, st, p);
    }
    if ((e = hipGetLastError()) != hipSuccess || p.B_out == 0 || p.layers == 0) return e;
    hipLaunchKernelGGL(baps_cache_fork_copy_kernel, dim3((unsigned)p.B_out, (unsigned)p.layers, kParts), dim3(256), 0, st, p);
    return hipGetLastError();
}

hipError_t launch_cache_compact(const CacheCompactParams& p, hipStream_t st)
{
    hipLaunchKernelGGL(baps_cache_compact_plan_kernel, dim3(1), dim3(kScan), 0, st, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    int ncu = 0;
    if ((e = cu_count(&ncu)) != hipSuccess) return e;
    const long long tg = (p.entries + 1023) / 1024;
    const int table_groups = (int)(tg > 256 ? 256 : tg);
    hipLaunchKernelGGL(baps_cache_compact_move_kernel, dim3((unsigned)(table_groups + 8 * ncu)), dim3(256), 0, st, p,
                       table_groups);
    return hipGetLastError();
}

}  // namespace baps
