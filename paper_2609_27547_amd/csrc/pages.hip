// Pages of an 8-bit KV cache (include/ebrl_kv8_pages.h): forks, releases,
// reservations with copies on write, compaction.
//
// What is decided goes by counts and ranks alone, never by the order in which
// workgroups run: the k-th need gets the k-th lowest free id.  A rank is the
// number of such pages in the chunks before a page's, which every workgroup adds
// up for itself from the counts that the launch before has written, and its rank
// in the chunk.  Atomics add and subtract whole numbers only.
#include <hip/hip_runtime.h>

#include "../../include/ebrl.h"
#include "../../include/ebrl_kv8_pages.h"
#include "kernels.h"

namespace ebrl {

constexpr int PG_CHUNK = 4096;      // refs that a workgroup of 256 threads counts
constexpr int PG_PIECE = 32768;     // bytes that a workgroup copies at a time
constexpr int PG_MAX_ROWS = 1 << 16;
constexpr int64_t PG_MAX_GROUPS = 1 << 23;

// ------------------------------------------------------- workgroup helpers --

// Sum over the workgroup's 256 threads, for each of them; `red`: 4 words.
EBRL_DEV int pg_sum(int v, int* red) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return red[0] + red[1] + red[2] + red[3];
}
// Sum of the values of the threads before this one; `red`: 4 words.
EBRL_DEV int pg_before(int v, int* red) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = v;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int t = __shfl_up(s, m, 64);
        if (lane >= m) s += t;
    }
    __syncthreads();
    if (lane == 63) red[wave] = s;
    __syncthreads();
    int base = 0;
    for (int w = 0; w < wave; ++w) base += red[w];
    return base + s - v;
}
// Sums of v[0 .. at) and of v[0 .. n).
EBRL_DEV int2 pg_prefix(const int* v, int at, int n, int* red) {
    int a = 0, b = 0;
    for (int i = threadIdx.x; i < n; i += 256) {
        const int x = v[i];
        b += x;
        if (i < at) a += x;
    }
    a = pg_sum(a, red);
    b = pg_sum(b, red);
    return make_int2(a, b);
}
// Whether v[0 .. n) holds x, for every thread of the workgroup.
EBRL_DEV bool pg_holds(const int* v, int n, int x) {
    bool found = false;
    for (int i = threadIdx.x; i < n; i += 256) found |= v[i] == x;
    return __syncthreads_or(found);
}

EBRL_DEV int pg_pages(int64_t tokens, int stride) {
    const int64_t p = (tokens + EBRL_KV8_PAGE - 1) / EBRL_KV8_PAGE;
    return tokens <= 0 ? 0 : p < stride ? (int)p : stride;
}
EBRL_DEV bool pg_page(int p, int num) { return (unsigned)p < (unsigned)num; }

// Copies piece `piece` of a page in one layer; `bytes`: of a page's codes, a
// multiple of 1024.  The first piece takes the scales along.
EBRL_DEV void pg_copy(const ebrl_kv8_pool& c, int from, int to, int layer, int piece, int bytes) {
    const char* src = (const char*)c.codes + (size_t)layer * c.layer_codes + (size_t)from * bytes;
    char* dst = (char*)c.codes + (size_t)layer * c.layer_codes + (size_t)to * bytes;
    const int end = min(bytes, (piece + 1) * PG_PIECE);
    for (int o = piece * PG_PIECE + threadIdx.x * 16; o < end; o += 4096)
        *reinterpret_cast<uint4*>(dst + o) = *reinterpret_cast<const uint4*>(src + o);
    if (piece == 0) {
        const int words = 2 * c.kv_heads;
        float* s = c.scales + (size_t)layer * c.layer_scales;
        for (int i = threadIdx.x; i < words; i += 256) s[(size_t)to * words + i] = s[(size_t)from * words + i];
    }
}

// ------------------------------------------------------------- fork, free --

__global__ __launch_bounds__(256) void pages_fork_kernel(ebrl_kv8_pool c, const int* src, const int* dst, const int* len,
                                                         int n)
{
    const int i = blockIdx.x, s = src[i], d = dst[i];
    if (!pg_page(s, c.table_rows) || !pg_page(d, c.table_rows)) return;
    if (pg_holds(dst, n, s) || pg_holds(dst, i, d)) return;
    const int keep = pg_pages(len[i], c.table_stride);
    const int* from = c.block_table + (size_t)s * c.table_stride;
    int* to = c.block_table + (size_t)d * c.table_stride;
    for (int j = threadIdx.x; j < c.table_stride; j += 256) {
        int p = j < keep ? from[j] : -1;
        if (!pg_page(p, c.num_blocks)) p = -1;
        const int old = to[j];
        if (p >= 0) atomicAdd(c.refs + p, 1);
        if (pg_page(old, c.num_blocks)) atomicSub(c.refs + old, 1);
        to[j] = p;
    }
}

// The exchange hands an entry's page to one of several threads that release it.
__global__ __launch_bounds__(256) void pages_free_kernel(ebrl_kv8_pool c, const int* seq, const int* keep)
{
    const int s = seq[blockIdx.x];
    if (!pg_page(s, c.table_rows)) return;
    int* row = c.block_table + (size_t)s * c.table_stride;
    for (int j = (keep ? pg_pages(keep[blockIdx.x], c.table_stride) : 0) + threadIdx.x; j < c.table_stride; j += 256) {
        const int p = atomicExch(row + j, -1);
        if (pg_page(p, c.num_blocks)) atomicSub(c.refs + p, 1);
    }
}

// ---------------------------------------------------------------- reserve --

// Workspace of a reservation: `chunks` counts of free pages; for each of n rows
// the number of pages that it needs and the page to copy (or -1); the local rank
// of each of its `pages` entries among those that need one (or -1); what is
// needed and free in all; the needed free ids.
struct PgReserve {
    int n, pages, chunks;
    int *free_count, *need, *copy, *rank, *total, *list;
};

__global__ __launch_bounds__(256) void pages_reserve_count_kernel(ebrl_kv8_pool c, const int* seq, const int* pos0,
                                                                  const int* count, int max_count, PgReserve w)
{
    __shared__ int red[4];
    if ((int)blockIdx.x < w.chunks) {
        const int p0 = blockIdx.x * PG_CHUNK;
        int free = 0;
        for (int p = threadIdx.x; p < PG_CHUNK; p += 256)
            if (p0 + p < c.num_blocks) free += c.refs[p0 + p] <= 0;
        free = pg_sum(free, red);
        if (threadIdx.x == 0) w.free_count[blockIdx.x] = free;
        return;
    }
    const int i = blockIdx.x - w.chunks, s = seq[i];
    const bool out = !pg_page(s, c.table_rows) || pg_holds(seq, i, s);
    const int pos = max(pos0[i], 0);
    const int64_t cap = (int64_t)c.table_stride * EBRL_KV8_PAGE;
    const int64_t end = min((int64_t)pos + min(max(count[i], 0), max_count), cap);
    const int j0 = pos / EBRL_KV8_PAGE;
    const int pages = out || end <= pos ? 0 : (int)((end + EBRL_KV8_PAGE - 1) / EBRL_KV8_PAGE) - j0;
    int base = 0;
    for (int q = 0; q < w.pages; q += 256) {
        const int j = q + threadIdx.x;
        bool need = false;
        if (j < pages) {
            const int p = c.block_table[(size_t)s * c.table_stride + j0 + j];
            const bool held = pg_page(p, c.num_blocks);
            need = !held || c.refs[p] > 1;
            if (j == 0) w.copy[i] = need && held && pos % EBRL_KV8_PAGE ? p : -1;
        } else if (j == 0) {
            w.copy[i] = -1;
        }
        const int at = pg_before(need, red);
        if (j < w.pages) w.rank[(size_t)i * w.pages + j] = need ? base + at : -1;
        base += pg_sum(need, red);
    }
    if (threadIdx.x == 0) w.need[i] = base;
}

// Free ids into the list, as many as are needed; needs of the rows before each.
__global__ __launch_bounds__(256) void pages_reserve_list_kernel(ebrl_kv8_pool c, int* lacking, PgReserve w)
{
    __shared__ int red[4];
    const int chunk = blockIdx.x;
    const int2 f = pg_prefix(w.free_count, chunk, w.chunks, red);
    const int needed = pg_prefix(w.need, 0, w.n, red).y;
    if (chunk == 0 && threadIdx.x == 0) {
        w.total[0] = needed;
        w.total[1] = f.y;
        *lacking = max(0, needed - f.y);
    }
    if (needed > f.y) return;
    int base = f.x;
    for (int q = 0; q < PG_CHUNK && base < needed; q += 256) {
        const int p = chunk * PG_CHUNK + q + threadIdx.x;
        const bool free = p < c.num_blocks && c.refs[p] <= 0;
        const int at = base + pg_before(free, red);
        if (free && at < needed) w.list[at] = p;
        base += pg_sum(free, red);
    }
}

// A row's new entries (piece 0 of layer 0) and the copy of its first page.
__global__ __launch_bounds__(256) void pages_reserve_kernel(ebrl_kv8_pool c, const int* seq, const int* pos0, int bytes,
                                                            int pieces, PgReserve w)
{
    __shared__ int red[4];
    const int i = blockIdx.x / pieces, piece = blockIdx.x % pieces, layer = blockIdx.y;
    if (w.total[0] > w.total[1]) return;
    const int from = w.copy[i];
    const bool entries = piece == 0 && layer == 0;
    if (w.need[i] == 0 || (!entries && from < 0)) return;
    const int before = pg_prefix(w.need, i, i, red).x;
    if (entries) {
        int* row = c.block_table + (size_t)seq[i] * c.table_stride + max(pos0[i], 0) / EBRL_KV8_PAGE;
        for (int j = threadIdx.x; j < w.pages; j += 256) {
            const int k = w.rank[(size_t)i * w.pages + j];
            if (k < 0) continue;
            const int p = w.list[before + k], old = row[j];
            if (pg_page(old, c.num_blocks)) atomicSub(c.refs + old, 1);
            c.refs[p] = 1;
            row[j] = p;
        }
    }
    if (from >= 0) pg_copy(c, from, w.list[before], layer, piece, bytes);
}

// ---------------------------------------------------------------- compact --

// Workspace of a compaction: counts of used pages by chunk; for each page its
// rank: of a free one below the end among those, of a used one past the end
// counted from the last of these, -1 for others; free ids below the end by rank;
// used ids past it, and their refs, by rank; {end, moves}.
struct PgCompact {
    int chunks;
    int *count, *rank, *hole, *mover, *mover_refs, *total;
};

__global__ __launch_bounds__(256) void pages_compact_count_kernel(ebrl_kv8_pool c, PgCompact w)
{
    __shared__ int red[4];
    const int p0 = blockIdx.x * PG_CHUNK;
    int used = 0;
    for (int p = threadIdx.x; p < PG_CHUNK; p += 256)
        if (p0 + p < c.num_blocks) used += c.refs[p0 + p] > 0;
    used = pg_sum(used, red);
    if (threadIdx.x == 0) w.count[blockIdx.x] = used;
}

__global__ __launch_bounds__(256) void pages_compact_list_kernel(ebrl_kv8_pool c, int* used, PgCompact w)
{
    __shared__ int red[4];
    const int p0 = blockIdx.x * PG_CHUNK;
    const int2 u = pg_prefix(w.count, blockIdx.x, w.chunks, red);
    const int end = u.y;
    int base = u.x;
    for (int q = 0; q < PG_CHUNK; q += 256) {
        const int p = p0 + q + threadIdx.x;
        const int r = p < c.num_blocks ? c.refs[p] : 0;
        const int before = base + pg_before(r > 0, red);   // used pages below p
        int rank = -1;
        if (p < end && r <= 0) {
            rank = p - before;
            w.hole[rank] = p;
        } else if (p >= end && r > 0) {
            rank = end - 1 - before;
            w.mover[rank] = p;
            w.mover_refs[rank] = r;
        }
        if (p < c.num_blocks) w.rank[p] = rank;
        // free pages below the end: as many as there are moves
        if (p == end - 1) w.total[1] = end - (before + (r > 0));
        base += pg_sum(r > 0, red);
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        w.total[0] = end;
        if (end == 0) w.total[1] = 0;
        *used = end;
    }
}

// Workgroups below `table_groups`: table and refs; the others: pages.
__global__ __launch_bounds__(256) void pages_compact_kernel(ebrl_kv8_pool c, int* new_table, int* new_refs, int bytes,
                                                            int pieces, int table_groups, PgCompact w)
{
    const int end = w.total[0], moves = w.total[1];
    if ((int)blockIdx.x < table_groups) {
        const int64_t entries = (int64_t)c.table_rows * c.table_stride, step = (int64_t)table_groups * 256;
        for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < entries; e += step) {
            int p = c.block_table[e];
            if (p >= end && p < c.num_blocks) {
                const int k = w.rank[p];
                if (k >= 0) p = w.hole[moves - 1 - k];
            }
            new_table[e] = p;
        }
        for (int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x; p < c.num_blocks; p += step) {
            int r = 0;
            if (p < end) {
                const int k = w.rank[p];
                r = k >= 0 ? w.mover_refs[moves - 1 - k] : c.refs[p];
            }
            new_refs[p] = r;
        }
        return;
    }
    const int64_t units = (int64_t)moves * c.layers * pieces;
    for (int64_t u = blockIdx.x - table_groups; u < units; u += gridDim.x - table_groups) {
        const int piece = (int)(u % pieces);
        const int64_t v = u / pieces;
        const int layer = (int)(v / moves), k = (int)(v % moves);
        pg_copy(c, w.mover[moves - 1 - k], w.hole[k], layer, piece, bytes);
    }
}

// ------------------------------------------------------------- the checks --

static bool pg_table_ok(const ebrl_kv8_pool* c) {
    return c && c->num_blocks >= 1 && c->num_blocks <= (1 << 30) && c->table_rows >= 1 && c->table_stride >= 1 &&
           c->table_stride < (1 << 27) && c->block_table && c->refs && (uintptr_t)c->block_table % 4 == 0 &&
           (uintptr_t)c->refs % 4 == 0;
}
static int64_t pg_bytes(const ebrl_kv8_pool* c) {
    return (int64_t)2 * c->kv_heads * EBRL_KV8_PAGE * c->head_dim;
}
static bool pg_shape_ok(const ebrl_kv8_pool* c) {
    return c && c->num_blocks >= 1 && c->num_blocks <= (1 << 30) && c->table_rows >= 1 && c->table_stride >= 1 &&
           c->table_stride < (1 << 27) && c->layers >= 1 && c->layers <= 65535 && c->kv_heads >= 1 &&
           c->kv_heads <= (1 << 17) && (c->head_dim == 64 || c->head_dim == 128);
}
static bool pg_pool_ok(const ebrl_kv8_pool* c) {
    if (!pg_shape_ok(c) || !pg_table_ok(c) || !c->codes || (uintptr_t)c->codes % 16 || !c->scales ||
        (uintptr_t)c->scales % 4)
        return false;
    return c->layers == 1 || (c->layer_codes % 16 == 0 && c->layer_codes >= 0 && c->layer_scales >= 0);
}
static int pg_chunks(const ebrl_kv8_pool* c) { return (c->num_blocks + PG_CHUNK - 1) / PG_CHUNK; }
static int pg_pieces(const ebrl_kv8_pool* c) { return (int)((pg_bytes(c) + PG_PIECE - 1) / PG_PIECE); }
// Pages that max_count tokens of a row touch at most.
static int64_t pg_most_pages(const ebrl_kv8_pool* c, int32_t max_count) {
    return std::min<int64_t>(((int64_t)max_count + 2 * EBRL_KV8_PAGE - 2) / EBRL_KV8_PAGE, c->table_stride);
}
static int64_t pg_reserve_words(const ebrl_kv8_pool* c, int64_t n, int64_t pages) {
    return pg_chunks(c) + 2 * n + n * pages + 2 + std::min<int64_t>(n * pages, c->num_blocks);
}
static int64_t pg_compact_words(const ebrl_kv8_pool* c) {
    return pg_chunks(c) + c->num_blocks + 3 * ((int64_t)c->num_blocks / 2 + 1) + 2;
}
static int pg_status() { return hipGetLastError() == hipSuccess ? EBRL_OK : EBRL_E_HIP; }

static bool pg_reserve_ok(const ebrl_kv8_pool* c, int32_t n, int32_t max_count) {
    return pg_shape_ok(c) && n >= 0 && n <= PG_MAX_ROWS && max_count >= 0 &&
           n * pg_most_pages(c, max_count) <= (1 << 30);
}

}  // namespace ebrl

using namespace ebrl;

extern "C" {

int ebrl_op_kv8_fork(const ebrl_kv8_pool* pool, const int32_t* src, const int32_t* dst, const int32_t* len, int32_t n,
                     void* stream) {
    if (!pg_table_ok(pool) || n < 0 || n > PG_MAX_ROWS) return EBRL_E_INVALID;
    if (n == 0) return EBRL_OK;
    if (!src || !dst || !len) return EBRL_E_INVALID;
    hipLaunchKernelGGL(pages_fork_kernel, dim3(n), dim3(256), 0, (hipStream_t)stream, *pool, src, dst, len, n);
    return pg_status();
}

int ebrl_op_kv8_free(const ebrl_kv8_pool* pool, const int32_t* seq, const int32_t* keep, int32_t n, void* stream) {
    if (!pg_table_ok(pool) || n < 0 || n > PG_MAX_ROWS) return EBRL_E_INVALID;
    if (n == 0) return EBRL_OK;
    if (!seq) return EBRL_E_INVALID;
    hipLaunchKernelGGL(pages_free_kernel, dim3(n), dim3(256), 0, (hipStream_t)stream, *pool, seq, keep);
    return pg_status();
}

int64_t ebrl_op_kv8_reserve_workspace(const ebrl_kv8_pool* pool, int32_t n, int32_t max_count) {
    if (!pg_reserve_ok(pool, n, max_count)) return EBRL_E_INVALID;
    return pg_reserve_words(pool, n, pg_most_pages(pool, max_count)) * 4;
}

int ebrl_op_kv8_reserve(const ebrl_kv8_pool* pool, const int32_t* seq, const int32_t* pos0, const int32_t* count,
                        int32_t n, int32_t max_count, int32_t* lacking, void* workspace, int64_t workspace_bytes,
                        void* stream) {
    if (!pg_reserve_ok(pool, n, max_count) || !pg_pool_ok(pool) || !lacking) return EBRL_E_INVALID;
    const int64_t pages = pg_most_pages(pool, max_count);
    const int pieces = pg_pieces(pool);
    const int64_t groups = std::max<int64_t>(1, (int64_t)n * pieces);
    if (groups * pool->layers > PG_MAX_GROUPS) return EBRL_E_INVALID;
    if (n > 0 && (!seq || !pos0 || !count)) return EBRL_E_INVALID;
    if (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < pg_reserve_words(pool, n, pages) * 4)
        return EBRL_E_INVALID;
    const hipStream_t s = (hipStream_t)stream;
    PgReserve w;
    w.n = n;
    w.pages = (int)pages;
    w.chunks = pg_chunks(pool);
    w.free_count = (int*)workspace;
    w.need = w.free_count + w.chunks;
    w.copy = w.need + n;
    w.total = w.copy + n;
    w.rank = w.total + 2;
    w.list = w.rank + (int64_t)n * pages;
    hipLaunchKernelGGL(pages_reserve_count_kernel, dim3(w.chunks + n), dim3(256), 0, s, *pool, seq, pos0, count, max_count, w);
    hipLaunchKernelGGL(pages_reserve_list_kernel, dim3(w.chunks), dim3(256), 0, s, *pool, lacking, w);
    if (n > 0)
        hipLaunchKernelGGL(pages_reserve_kernel, dim3((unsigned)groups, pool->layers), dim3(256), 0, s, *pool, seq, pos0,
                           (int)pg_bytes(pool), pieces, w);
    return pg_status();
}

int64_t ebrl_op_kv8_compact_workspace(const ebrl_kv8_pool* pool) {
    return pg_shape_ok(pool) ? pg_compact_words(pool) * 4 : EBRL_E_INVALID;
}

int ebrl_op_kv8_compact(const ebrl_kv8_pool* pool, int32_t* new_table, int32_t* new_refs, int32_t* used,
                        void* workspace, int64_t workspace_bytes, void* stream) {
    if (!pg_pool_ok(pool) || !new_table || !new_refs || !used) return EBRL_E_INVALID;
    if (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < pg_compact_words(pool) * 4) return EBRL_E_INVALID;
    const hipStream_t s = (hipStream_t)stream;
    const int64_t half = pool->num_blocks / 2 + 1;
    PgCompact w;
    w.chunks = pg_chunks(pool);
    w.count = (int*)workspace;
    w.rank = w.count + w.chunks;
    w.hole = w.rank + pool->num_blocks;
    w.mover = w.hole + half;
    w.mover_refs = w.mover + half;
    w.total = w.mover_refs + half;
    const int pieces = pg_pieces(pool);
    const int64_t entries = std::max<int64_t>((int64_t)pool->table_rows * pool->table_stride, pool->num_blocks);
    const int table_groups = (int)std::min<int64_t>(256, (entries + 1023) / 1024);
    const int64_t most = (int64_t)(pool->num_blocks / 2) * pool->layers * pieces;
    const int copy_groups = (int)std::min<int64_t>(2048, most);
    hipLaunchKernelGGL(pages_compact_count_kernel, dim3(w.chunks), dim3(256), 0, s, *pool, w);
    hipLaunchKernelGGL(pages_compact_list_kernel, dim3(w.chunks), dim3(256), 0, s, *pool, used, w);
    hipLaunchKernelGGL(pages_compact_kernel, dim3(table_groups + copy_groups), dim3(256), 0, s, *pool, new_table,
                       new_refs, (int)pg_bytes(pool), pieces, table_groups, w);
    return pg_status();
}

}  // extern "C"
