// The upkeep of a paged cache (include/kv_cache.h): pages given out, given back, shared, moved together, for gfx950 (MI355X).
//
// Contents are moved by as many workgroups as there is work for, a plain stream bound by memory.  Who gets which page is decided by one
// workgroup: it scans `ref` in order, 4096 pages a step, so the lowest free page is a matter of a running count and results do not
// depend on who comes first.  Counts are changed by integer atomics, whose order does not matter either.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gfx950_prims.h"
#include "paged_launch.h"

namespace {

constexpr int PLAN = 1024;                      // threads of the deciding workgroup
constexpr int PER = 4;                          // pages (rows of a list) that a thread takes at a time

// Tokens of a row, within what its table row can hold, and the pages that they fill.
__device__ __forceinline__ int tokens_of(const kv_book& b, int len) { return min(max(len, 0), b.table_width * b.page_size); }
__device__ __forceinline__ int pages_of(const kv_book& b, int len) { return (int)(((unsigned)tokens_of(b, len) + b.page_size - 1) / b.page_size); }

// Exclusive prefix sum over the workgroup; `total` is the sum.  Every thread calls it.
__device__ __forceinline__ int prefix(int x, int& total)
{
    __shared__ int sums[PLAN / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int y = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int z = __shfl_up(y, d);
        if (lane >= d) y += z;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = y;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < PLAN / 64; ++w) {
        if (w < wave) before += sums[w];
        total += sums[w];
    }
    return before + y - x;
}

// Calls give(k, page) for the k-th free page, k < want, from the threads that found them; returns how many there were.
template <typename Give> __device__ __forceinline__ int give_free(const int* ref, int pages, int want, Give give)
{
    int done = 0;
    for (int p0 = 0; p0 < pages && done < want; p0 += PLAN * PER) {
        const int p = p0 + threadIdx.x * PER;
        bool free[PER];
        int n = 0, total;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            free[i] = p + i < pages && ref[min(p + i, pages - 1)] == 0;
            n += free[i];
        }
        int k = done + prefix(n, total);
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (free[i]) {
                if (k < want) give(k, p + i);
                ++k;
            }
        done += total;
    }
    return min(done, want);
}

// Prefix sums of a list's wants in the LDS: before[i] of element i, before[n] the sum.
template <typename Want> __device__ __forceinline__ void sum_list(int* before, int n, Want want)
{
    int done = 0;
    for (int i0 = 0; i0 < n; i0 += PLAN) {
        const int i = i0 + threadIdx.x;
        int total;
        const int at = done + prefix(i < n ? want(i) : 0, total);
        if (i < n) before[i] = at;
        done += total;
    }
    if (threadIdx.x == 0) before[n] = done;
    __syncthreads();
}
// The element that the k-th wanted page goes to.
__device__ __forceinline__ int whose(const int* before, int n, int k)
{
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (before[mid] <= k) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__global__ __launch_bounds__(PLAN)
void reserve_kernel(kv_book b, const int* list, const int* new_len, int n, int* missing)
{
    extern __shared__ int before[];
    auto held = [&](int r) { return pages_of(b, b.kv_len[r]); };
    sum_list(before, n, [&](int i) {
        const int r = list[i];
        return (unsigned)r < (unsigned)b.rows ? max(0, pages_of(b, new_len[i]) - held(r)) : 0;
    });
    const int want = before[n];
    const int got = give_free(b.ref, b.pages, want, [&](int k, int page) {
        const int i = whose(before, n, k), r = list[i];
        b.table[(long long)r * b.table_stride + held(r) + k - before[i]] = page;
        b.ref[page] = 1;
    });
    for (int k = got + threadIdx.x; k < want; k += PLAN) {
        const int i = whose(before, n, k), r = list[i];
        b.table[(long long)r * b.table_stride + held(r) + k - before[i]] = -1;
    }
    __syncthreads();                            // (lengths change only now)
    for (int i = threadIdx.x; i < n; i += PLAN) {
        const int r = list[i];
        if ((unsigned)r < (unsigned)b.rows && tokens_of(b, new_len[i]) > b.kv_len[r]) b.kv_len[r] = tokens_of(b, new_len[i]);
    }
    if (threadIdx.x == 0) *missing = want - got;
}

__global__ __launch_bounds__(256)
void free_kernel(kv_book b, const int* list)
{
    const int r = list[blockIdx.x];
    if ((unsigned)r >= (unsigned)b.rows) return;
    const int n = pages_of(b, b.kv_len[r]);
    int* const row = b.table + (long long)r * b.table_stride;
    // (the exchange lets one of two workgroups with the same row give a page back)
    for (int j = threadIdx.x; j < n; j += 256) {
        const int page = atomicExch(&row[j], -1);
        if ((unsigned)page < (unsigned)b.pages) atomicSub(&b.ref[page], 1);
    }
    __syncthreads();
    if (threadIdx.x == 0) b.kv_len[r] = 0;
}

// Part `part` of `parts` of a page's contents by a workgroup, 16 bytes a lane, UNROLL of them under way (256 pages of 1 MiB in 8 layers moving together, 525 MB read and
// written: 120 / 119 / 118 / 115 us with 1 / 2 / 4 / 8).
constexpr int UNROLL = 8;
__device__ __forceinline__ void copy_page(const PageCopy& c, char* base, int layer, long long src, long long dst, int part, int parts)
{
    const int cols = c.row_bytes / 16, all = c.heads * c.page_size * cols, per = (all + parts - 1) / parts, end = min(all, (part + 1) * per);
    const char* const from = base + layer * c.layer + src * c.page;
    char* const to = base + layer * c.layer + dst * c.page;
    const bool heads_inside = c.head < c.token;
    for (int i0 = part * per + threadIdx.x; i0 < end; i0 += 256 * UNROLL) {
        long long at[UNROLL];
        u32x4 w[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int i = min(i0 + u * 256, end - 1);
            if (c.solid) {
                at[u] = i * 16ll;
            } else {
                const int col = i % cols, r = i / cols, h = heads_inside ? r % c.heads : r / c.page_size, t = heads_inside ? r / c.heads : r % c.page_size;
                at[u] = h * c.head + t * c.token + col * 16;
            }
            w[u] = *reinterpret_cast<const u32x4*>(from + at[u]);
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
            if (i0 + u * 256 < end) *reinterpret_cast<u32x4*>(to + at[u]) = w[u];
    }
}

// The last page of row s, of len tokens, if it is not full and is there, else -1.  (Where it is not there, the continuation has none either: a page given out in its
// place would show what its last owner left in it.)
__device__ __forceinline__ int part_page(const kv_book& b, int s, int len)
{
    if (len % b.page_size == 0) return -1;
    const int page = b.table[(long long)s * b.table_stride + len / b.page_size];
    return (unsigned)page < (unsigned)b.pages ? page : -1;
}

__global__ __launch_bounds__(PLAN)
void fork_plan_kernel(kv_book b, const int* src, const int* dst, int n, int* missing)
{
    extern __shared__ int before[];
    sum_list(before, n, [&](int i) {
        const int s = src[i], d = dst[i];
        return (unsigned)s < (unsigned)b.rows && (unsigned)d < (unsigned)b.rows && s != d && part_page(b, s, tokens_of(b, b.kv_len[s])) >= 0 ? 1 : 0;
    });
    const int want = before[n];
    auto place = [&](int k) -> int& {
        const int i = whose(before, n, k);
        return b.table[(long long)dst[i] * b.table_stride + tokens_of(b, b.kv_len[src[i]]) / b.page_size];
    };
    const int got = give_free(b.ref, b.pages, want, [&](int k, int page) {
        place(k) = page;
        b.ref[page] = 1;
    });
    for (int k = got + threadIdx.x; k < want; k += PLAN) place(k) = -1;
    if (threadIdx.x == 0) *missing = want - got;
}

// blockIdx.y: pair.  blockIdx.x 0: the table row; 1 ...: layer, keys or values, part of the last page.
__global__ __launch_bounds__(256)
void fork_kernel(PageCopy c, kv_book b, const int* src, const int* dst, int parts)
{
    const int s = src[blockIdx.y], d = dst[blockIdx.y];
    if ((unsigned)s >= (unsigned)b.rows || (unsigned)d >= (unsigned)b.rows || s == d) return;
    const int len = tokens_of(b, b.kv_len[s]), full = len / b.page_size, part = part_page(b, s, len);
    const int* const from = b.table + (long long)s * b.table_stride;
    int* const to = b.table + (long long)d * b.table_stride;
    if (blockIdx.x == 0) {
        for (int j = threadIdx.x; j < b.table_width; j += 256) {
            if (j == full && part >= 0) continue;    // (the plan has put it there)
            const int page = j < full ? from[j] : -1;
            to[j] = page;
            if ((unsigned)page < (unsigned)b.pages) atomicAdd(&b.ref[page], 1);
        }
        if (threadIdx.x == 0) b.kv_len[d] = len;
        return;
    }
    if (part < 0) return;
    const int now = to[full];
    if ((unsigned)now >= (unsigned)b.pages) return;
    int id = blockIdx.x - 1;
    const int p = id % parts;
    id /= parts;
    copy_page(c, id & 1 ? c.v : c.k, id >> 1, part, now, p, parts);
}

__global__ __launch_bounds__(256)
void copy_pages_kernel(PageCopy c, const int* src, const int* dst, int parts)
{
    const int s = src[blockIdx.y], d = dst[blockIdx.y];
    if ((unsigned)s >= (unsigned)c.pages || (unsigned)d >= (unsigned)c.pages || s == d) return;
    int id = blockIdx.x;
    const int p = id % parts;
    id /= parts;
    copy_page(c, id & 1 ? c.v : c.k, id >> 1, s, d, p, parts);
}

// Workspace of kv_compact: [0] moves, [1] pages in use, from [4] the new number of every page (of those from [1] on; -1: it stays), then the pairs (from, to).
__global__ __launch_bounds__(PLAN)
void compact_plan_kernel(kv_book b, int* ws)
{
    __shared__ int s_live;
    if (threadIdx.x == 0) s_live = 0;
    __syncthreads();
    int mine = 0;
    for (int p = threadIdx.x; p < b.pages; p += PLAN) mine += b.ref[p] > 0;
    atomicAdd(&s_live, mine);
    __syncthreads();
    const int live = s_live;
    int* const moved = ws + 4;
    int* const pairs = moved + b.pages;
    int holes = 0, movers = 0;
    for (int p0 = 0; p0 < b.pages; p0 += PLAN * PER) {
        const int p = p0 + threadIdx.x * PER;
        int kind[PER], n = 0, total;            // 1: a hole below `live`, 2: in use above
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const bool used = b.ref[min(p + i, b.pages - 1)] > 0;
            kind[i] = p + i >= b.pages || used == (p + i < live) ? 0 : used ? 2 : 1;
            n += kind[i] == 1 ? 1 : kind[i] == 2 ? 1 << 16 : 0;
            if (p + i >= live && p + i < b.pages && !used) moved[p + i] = -1;
        }
        const int at = prefix(n, total);        // (both counts in one sum: at most 4096 each)
        int hole = holes + (at & 0xffff), mover = movers + (at >> 16);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (kind[i] == 1) pairs[2 * hole++ + 1] = p + i;
            if (kind[i] == 2) pairs[2 * mover++] = p + i;
        }
        holes += total & 0xffff;
        movers += total >> 16;
    }
    __syncthreads();                            // (as many holes as movers: `live` pages are in use)
    for (int i = threadIdx.x; i < holes; i += PLAN) {
        const int from = pairs[2 * i], to = pairs[2 * i + 1];
        moved[from] = to;
        b.ref[to] = b.ref[from];
        b.ref[from] = 0;
    }
    if (threadIdx.x == 0) {
        ws[0] = holes;
        ws[1] = live;
    }
}

// The first `table_blocks` workgroups renumber table entries, the others move contents.
__global__ __launch_bounds__(256)
void compact_kernel(PageCopy c, kv_book b, const int* ws, int table_blocks, int parts)
{
    const int moves = ws[0], live = ws[1];
    if (moves == 0) return;
    const int* const moved = ws + 4;
    const int* const pairs = moved + b.pages;
    if ((int)blockIdx.x < table_blocks) {
        for (int r = blockIdx.x; r < b.rows; r += table_blocks) {
            int* const row = b.table + (long long)r * b.table_stride;
            const int n = pages_of(b, b.kv_len[r]);
            for (int j = threadIdx.x; j < n; j += 256) {
                const int page = row[j];
                // (-1: a page without a holder that stands in a table all the same)
                if (page >= live && page < b.pages && moved[page] >= 0) row[j] = moved[page];
            }
        }
        return;
    }
    const long long all = (long long)moves * c.layers * 2 * parts;
    for (long long id = blockIdx.x - table_blocks; id < all; id += gridDim.x - table_blocks) {
        const int p = (int)(id % parts);
        long long rest = id / parts;
        const int what = (int)(rest % (2 * c.layers));
        const int* const pair = pairs + rest / (2 * c.layers) * 2;
        copy_page(c, what & 1 ? c.v : c.k, what >> 1, pair[0], pair[1], p, parts);
    }
}

// Workgroups that share a page of one layer: one for every 32 KiB.
int parts_of(const PageCopy& c)
{
    const long long bytes = (long long)c.heads * c.page_size * c.row_bytes;
    return (int)((bytes + (32 << 10) - 1) / (32 << 10));
}

int go(const void* kern, dim3 grid, int threads, void** args, int smem, void* stream)
{
    return hipLaunchKernel(kern, grid, dim3(threads), args, smem, (hipStream_t)stream) == hipSuccess ? 0 : -1;
}

}  // namespace

int kv_reserve_launch(const kv_book& b, const int* list, const int* new_len, int n, int* missing, void* stream)
{
    kv_book book = b;
    void* args[] = {&book, &list, &new_len, &n, &missing};
    return go(reinterpret_cast<const void*>(reserve_kernel), dim3(1), PLAN, args, (n + 1) * 4, stream);
}

int kv_free_launch(const kv_book& b, const int* list, int n, void* stream)
{
    kv_book book = b;
    void* args[] = {&book, &list};
    return go(reinterpret_cast<const void*>(free_kernel), dim3(n), 256, args, 0, stream);
}

int kv_fork_launch(const PageCopy& c, const kv_book& b, const int* src, const int* dst, int n, int* missing, void* stream)
{
    kv_book book = b;
    PageCopy copy = c;
    int parts = parts_of(c);
    void* plan[] = {&book, &src, &dst, &n, &missing};
    if (go(reinterpret_cast<const void*>(fork_plan_kernel), dim3(1), PLAN, plan, (n + 1) * 4, stream) != 0) return -1;
    if (n == 0) return 0;
    void* args[] = {&copy, &book, &src, &dst, &parts};
    return go(reinterpret_cast<const void*>(fork_kernel), dim3(1 + c.layers * 2 * parts, n), 256, args, 0, stream);
}

int kv_compact_launch(const PageCopy& c, const kv_book& b, int* workspace, void* stream)
{
    kv_book book = b;
    PageCopy copy = c;
    int parts = parts_of(c), table_blocks = b.rows < 256 ? b.rows : 256;
    void* plan[] = {&book, &workspace};
    if (go(reinterpret_cast<const void*>(compact_plan_kernel), dim3(1), PLAN, plan, 0, stream) != 0) return -1;
    const long long most = (long long)(b.pages / 2) * c.layers * 2 * parts;
    const int movers = most < 4096 ? (most < 1 ? 1 : (int)most) : 4096;
    void* args[] = {&copy, &book, &workspace, &table_blocks, &parts};
    return go(reinterpret_cast<const void*>(compact_kernel), dim3(table_blocks + movers), 256, args, 0, stream);
}

int kv_copy_pages_launch(const PageCopy& c, const int* src, const int* dst, int n, void* stream)
{
    PageCopy copy = c;
    int parts = parts_of(c);
    void* args[] = {&copy, &src, &dst, &parts};
    return go(reinterpret_cast<const void*>(copy_pages_kernel), dim3(c.layers * 2 * parts, n), 256, args, 0, stream);
}
