// Pages of an 8-bit KV cache (include/ebrl_kv8_pages.h): forks, releases,
// reservations with copies on write, compaction.
//
// What is decided goes by counts and ranks alone, never by the order in which
// workgroups run: the k-th need gets the k-th lowest free id.  A rank is the
// number of such pages in the chunks before a page's, which every workgroup adds
// up for itself from the counts that the launch before has written, and its rank
// in the chunk.  Atomics add and subtract whole numbers only.
//
// Bound by launches and latencies where little is copied (8 branches of two prefixes:
// 2.5 us a release, 3.6 a fork, 4.4 each of the two launches of a reservation), else by
// memory: 256 branches of 1 MB pages 53 us, writes at 4.8 TB/s (their 16 source pages
// stay in the caches: with the loads left out it takes as long); 900 moves of 576 KB 205
// us, 5.2 TB/s read and written, where a large copy makes 4.8.
#include <hip/hip_runtime.h>

#include "../../include/ebrl.h"
#include "../../include/ebrl_kv8_pages.h"
#include "kernels.h"

namespace ebrl {

constexpr int PG_CHUNK = 4096;      // refs that a workgroup counts: sixteen neighbours a thread
constexpr int PG_PIECE = 16384;     // bytes that a workgroup copies at a time: four loads a thread
constexpr int PG_MAX_ROWS = 1 << 16;
constexpr int64_t PG_MAX_GROUPS = 1 << 23;

// ------------------------------------------------------- workgroup helpers --

// Of each thread's value: the sum of those of the threads before it, and of all.
// `red`: a word for each wave.
template <int WAVES> EBRL_DEV int2 pg_scan(int v, int* red) {
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
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const int t = red[w];
        all += t;
        if (w < wave) before += t;
    }
    return make_int2(before + s - v, all);
}
// Sums of v[0 .. at) and of v[0 .. n), for workgroups of 256.
EBRL_DEV int2 pg_prefix(const int* v, int at, int n, int* red) {
    int a = 0, b = 0;
    for (int i = threadIdx.x; i < n; i += 256) {
        const int x = v[i];
        b += x;
        if (i < at) a += x;
    }
    return make_int2(pg_scan<4>(a, red).y, pg_scan<4>(b, red).y);
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

// Which of pages p .. p + 15 are in use, a bit each; those past the pool are not.
EBRL_DEV unsigned pg_used16(const ebrl_kv8_pool& c, int p) {
    unsigned m = 0;
    if (p + 16 <= c.num_blocks && (uintptr_t)c.refs % 16 == 0) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int4 r = *reinterpret_cast<const int4*>(c.refs + p + 4 * k);
            m |= ((r.x > 0 ? 1u : 0u) | (r.y > 0 ? 2u : 0u) | (r.z > 0 ? 4u : 0u) | (r.w > 0 ? 8u : 0u)) << 4 * k;
        }
    } else {
        for (int k = 0; k < 16 && p + k < c.num_blocks; ++k) m |= (c.refs[p + k] > 0 ? 1u : 0u) << k;
    }
    return m;
}
// Which of them exist.
EBRL_DEV unsigned pg_there16(const ebrl_kv8_pool& c, int p) {
    const int n = c.num_blocks - p;
    return n >= 16 ? 0xFFFFu : n > 0 ? (1u << n) - 1 : 0u;
}

// Copies piece `piece` of a page in one layer; `bytes`: of a page's codes, a
// multiple of 1024.  The first piece takes the scales along.  Bound by memory: a
// thread's loads are in flight before its first store, and what is written is not read
// again here (900 pages of 32 KB in 18 layers 191 us with non-temporal loads and stores,
// 209 with plain ones; 256 copies of 16 pages in 32 layers 54 us with plain loads, whose
// pages stay in the caches, 82 without).  ONCE: no other copy reads the same page.
template <bool ONCE> EBRL_DEV void pg_copy(const ebrl_kv8_pool& c, int from, int to, int layer, int piece, int bytes) {
    constexpr int N = PG_PIECE / 4096;
    const size_t base = (size_t)layer * c.layer_codes + (size_t)piece * PG_PIECE;
    const char* src = (const char*)c.codes + base + (size_t)from * bytes + threadIdx.x * 16;
    char* dst = (char*)c.codes + base + (size_t)to * bytes + threadIdx.x * 16;
    auto load = [](const char* p) {
        const u32x4* q = reinterpret_cast<const u32x4*>(p);
        return ONCE ? __builtin_nontemporal_load(q) : *q;
    };
    const int left = bytes - piece * PG_PIECE;
    if (left >= PG_PIECE) {
        u32x4 v[N];
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = load(src + k * 4096);
#pragma unroll
        for (int k = 0; k < N; ++k) __builtin_nontemporal_store(v[k], reinterpret_cast<u32x4*>(dst + k * 4096));
    } else {
        for (int o = 0; o + (int)threadIdx.x * 16 < left; o += 4096)
            __builtin_nontemporal_store(load(src + o), reinterpret_cast<u32x4*>(dst + o));
    }
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

// A reservation's numbers in the workspace.
struct PgReserve {
    int n, pages, chunks;
    int* free_count;    // [chunks] free pages of each
    int* need;          // [n] pages that row i needs
    int* before;        // [n] ... and the rows before it
    int* copy;          // [n] the page to copy, or -1
    int* total;         // pages needed and free in all
    int* rank;          // [n][pages] an entry's number among those of its row that need a page, or -1
    int* list;          // the free ids, as many as are needed
};
// Entries of row i that the call looks at: `pages` of them from j0 on, none if it is
// left out.
struct PgSpan { int row, pos, j0, pages; };
EBRL_DEV PgSpan pg_span(const ebrl_kv8_pool& c, const int* seq, const int* pos0, const int* count, int max_count, int i) {
    PgSpan r;
    r.row = seq[i];
    r.pos = max(pos0[i], 0);
    r.j0 = r.pos / EBRL_KV8_PAGE;
    const int64_t end = min((int64_t)r.pos + min(max(count[i], 0), max_count), (int64_t)c.table_stride * EBRL_KV8_PAGE);
    r.pages = !pg_page(r.row, c.table_rows) || end <= r.pos ? 0 : (int)((end + EBRL_KV8_PAGE - 1) / EBRL_KV8_PAGE) - r.j0;
    return r;
}
// Whether entry j of the span needs a page; the first one tells what to copy.
EBRL_DEV bool pg_need(const ebrl_kv8_pool& c, const PgSpan& r, int j, int* copy) {
    bool need = false;
    int from = -1;
    if (j < r.pages) {
        const int p = c.block_table[(size_t)r.row * c.table_stride + r.j0 + j];
        const bool held = pg_page(p, c.num_blocks);
        need = !held || c.refs[p] > 1;
        if (need && held && r.pos % EBRL_KV8_PAGE) from = p;
    }
    if (j == 0) *copy = from;
    return need;
}

// Small calls (PG_SMALL_*): everything that is decided, in one workgroup of sixteen
// waves: a row and then an entry a thread, ids a page a lane.  Bound by latency: 256
// rows of 5 entries 21.7 us with a row a wave at a time, 9.5 so.
constexpr int PG_SMALL_ROWS = 1024, PG_SMALL_POOL = 1 << 16, PG_SMALL_ENTRIES = 1 << 14;

// Pages wave `wave` of sixteen looks at, 64 at a time: first and last of them.
EBRL_DEV int2 pg_wave_pages(int num, int wave) {
    const int per = (num + 1023) / 1024 * 64;
    return make_int2(min(num, wave * per), min(num, (wave + 1) * per));
}
// Number of lanes below this one whose bit is set.
EBRL_DEV int pg_below(uint64_t m) {
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}
// Pages in use among r.x .. r.y - 1, for a whole wave.
EBRL_DEV int pg_wave_used(const ebrl_kv8_pool& c, int2 r) {
    int used = 0;
    const int lane = threadIdx.x & 63;
    for (int p = r.x; p < r.y; p += 512) {
        int v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = c.refs[min(p + k * 64 + lane, r.y - 1)];
#pragma unroll
        for (int k = 0; k < 8; ++k) used += (int)__popcll(__ballot(p + k * 64 + lane < r.y && v[k] > 0));
    }
    return used;
}

__global__ __launch_bounds__(1024) void pages_reserve_small_kernel(ebrl_kv8_pool c, const int* seq, const int* pos0,
                                                                   const int* count, int max_count, int* lacking,
                                                                   PgReserve w)
{
    __shared__ int s_seq[PG_SMALL_ROWS], red[16];
    __shared__ bool s_again[PG_SMALL_ROWS];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int2 mine = pg_wave_pages(c.num_blocks, wave);
    if (tid < w.n) {
        s_seq[tid] = seq[tid];
        s_again[tid] = false;
        w.before[tid] = 0;      // ranks count through all rows
    }
    // free pages of the waves before this one, and of all
    const int free = mine.y - mine.x - pg_wave_used(c, mine);
    const int2 f = pg_scan<16>(lane == 0 ? free : 0, red);
    const int free_before = __builtin_amdgcn_readfirstlane(f.x);
    __syncthreads();
    // rows that an earlier number names too: several threads a row where rows are few
    const int span = (w.n + 63) & ~63, parts = 1024 / max(span, 64), i0 = tid % max(span, 64);
    if (i0 < w.n) {
        bool again = false;
        for (int k = tid / max(span, 64); k < i0; k += parts) again |= s_seq[k] == s_seq[i0];
        if (again) s_again[i0] = true;
    }
    __syncthreads();
    int needed = 0;
    for (int q = 0; q < w.n * w.pages; q += 1024) {
        const int e = q + tid, i = min(e / w.pages, w.n - 1), j = e - i * w.pages;
        bool need = false;
        if (e < w.n * w.pages) {
            PgSpan r = pg_span(c, seq, pos0, count, max_count, i);
            if (s_again[i]) r.pages = 0;
            need = pg_need(c, r, j, w.copy + i);
        }
        const int2 at = pg_scan<16>(need, red);
        if (e < w.n * w.pages) w.rank[e] = need ? needed + at.x : -1;
        needed += at.y;
    }
    if (tid == 0) {
        w.total[0] = needed;
        w.total[1] = f.y;
        *lacking = max(0, needed - f.y);
    }
    int at = free_before;
    for (int q = mine.x; q < mine.y && at < needed; q += 256) {
        int v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = c.refs[min(q + k * 64 + lane, mine.y - 1)];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int p = q + k * 64 + lane;
            const bool is = p < mine.y && v[k] <= 0;
            const uint64_t m = __ballot(is);
            const int to = at + pg_below(m);
            if (is && to < needed) w.list[to] = p;
            at += (int)__popcll(m);
        }
    }
}

// The others: counts, by chunks of pages and by rows ...
__global__ __launch_bounds__(256) void pages_reserve_count_kernel(ebrl_kv8_pool c, const int* seq, const int* pos0,
                                                                  const int* count, int max_count, PgReserve w)
{
    __shared__ int red[4];
    if ((int)blockIdx.x < w.chunks) {
        const int p = blockIdx.x * PG_CHUNK + threadIdx.x * 16;
        const int free = pg_scan<4>(__popc(pg_used16(c, p) ^ pg_there16(c, p)), red).y;
        if (threadIdx.x == 0) w.free_count[blockIdx.x] = free;
        return;
    }
    const int i = blockIdx.x - w.chunks;
    PgSpan r = pg_span(c, seq, pos0, count, max_count, i);
    if (pg_holds(seq, i, r.row)) r.pages = 0;
    int base = 0;
    for (int q = 0; q < w.pages; q += 256) {
        const int j = q + threadIdx.x;
        const bool need = pg_need(c, r, j, w.copy + i);
        const int2 at = pg_scan<4>(need, red);
        if (j < w.pages) w.rank[(size_t)i * w.pages + j] = need ? base + at.x : -1;
        base += at.y;
    }
    if (threadIdx.x == 0) w.need[i] = base;
}
// ... then free ids into the list, as many as are needed, and (the last workgroup) the
// needs of the rows before each.
__global__ __launch_bounds__(256) void pages_reserve_list_kernel(ebrl_kv8_pool c, int* lacking, PgReserve w)
{
    __shared__ int red[4];
    const int chunk = blockIdx.x;
    if (chunk == w.chunks) {
        int base = 0;
        for (int q = 0; q < w.n; q += 256) {
            const int i = q + threadIdx.x;
            const int2 r = pg_scan<4>(i < w.n ? w.need[i] : 0, red);
            if (i < w.n) w.before[i] = base + r.x;
            base += r.y;
        }
        return;
    }
    const int p = chunk * PG_CHUNK + threadIdx.x * 16;
    unsigned m = pg_used16(c, p) ^ pg_there16(c, p);
    const int2 f = pg_prefix(w.free_count, chunk, w.chunks, red);
    const int needed = pg_prefix(w.need, 0, w.n, red).y;
    if (chunk == 0 && threadIdx.x == 0) {
        w.total[0] = needed;
        w.total[1] = f.y;
        *lacking = max(0, needed - f.y);
    }
    int at = f.x + pg_scan<4>(__popc(m), red).x;
    for (; m && at < needed; m &= m - 1, ++at) w.list[at] = p + __builtin_ctz(m);
}

// A row's new entries (piece 0 of the first layers) and the copy of its first page, in
// `step` layers.
__global__ __launch_bounds__(256) void pages_reserve_kernel(ebrl_kv8_pool c, const int* seq, const int* pos0, int bytes,
                                                            int pieces, int step, PgReserve w)
{
    const int i = blockIdx.x / pieces, piece = blockIdx.x % pieces, layer = blockIdx.y * step;
    const int from = w.copy[i], before = w.before[i], first = w.rank[(size_t)i * w.pages];
    const bool entries = piece == 0 && layer == 0;
    if (w.total[0] > w.total[1] || (!entries && from < 0)) return;
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
    if (from < 0) return;
    const int to = w.list[before + first];
    const int end = min(layer + step, c.layers);
    for (int l = layer; l < end; ++l) pg_copy<false>(c, from, to, l, piece, bytes);
}

// ---------------------------------------------------------------- compact --

// A compaction's numbers in the workspace.
struct PgCompact {
    int chunks;
    int* count;         // [chunks] used pages of each
    int* rank;          // [num_blocks] of a free page below the end: its number among those; of a used one
                        // past it: its number, from the last of those; -1 of others
    int* hole;          // the free ids below the end
    int* mover;         // the used ones past it, the last first
    int* mover_refs;    // ... their refs
    int* total;         // the end (pages in use) and the moves
};
// Sixteen pages' ranks and places in the lists; m: which are in use, `before`: how many
// below them are.
EBRL_DEV void pg_place16(const ebrl_kv8_pool& c, const PgCompact& w, int p, unsigned m, int before, int end) {
    const unsigned there = pg_there16(c, p);
#pragma unroll 1
    for (int k = 0; k < 16; ++k) {
        if (!(there >> k & 1)) break;
        const bool used = m >> k & 1;
        int rank = -1;
        if (p + k < end && !used) {
            rank = p + k - before;
            w.hole[rank] = p + k;
        } else if (p + k >= end && used) {
            rank = end - 1 - before;
            w.mover[rank] = p + k;
            w.mover_refs[rank] = c.refs[p + k];
        }
        w.rank[p + k] = rank;
        before += used;
        // free pages below the end: as many as there are moves
        if (p + k == end - 1) w.total[1] = end - before;
    }
}

// Small pools: in one workgroup, a page a lane.
__global__ __launch_bounds__(1024) void pages_compact_small_kernel(ebrl_kv8_pool c, int* used, PgCompact w)
{
    __shared__ int red[16];
    const int tid = threadIdx.x, lane = tid & 63;
    const int2 mine = pg_wave_pages(c.num_blocks, tid >> 6);
    const int of_wave = pg_wave_used(c, mine);
    const int2 u = pg_scan<16>(lane == 0 ? of_wave : 0, red);
    const int end = u.y;
    if (tid == 0) {
        w.total[0] = end;
        if (end == 0) w.total[1] = 0;
        *used = end;
    }
    int below = __builtin_amdgcn_readfirstlane(u.x);
    for (int q = mine.x; q < mine.y; q += 256) {
        int v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = c.refs[min(q + k * 64 + lane, mine.y - 1)];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int p = q + k * 64 + lane;
            const bool is = p < mine.y && v[k] > 0;
            const uint64_t m = __ballot(is);
            const int before = below + pg_below(m);
            below += (int)__popcll(m);
            if (p >= mine.y) continue;
            int rank = -1;
            if (p < end && !is) {
                rank = p - before;
                w.hole[rank] = p;
            } else if (p >= end && is) {
                rank = end - 1 - before;
                w.mover[rank] = p;
                w.mover_refs[rank] = v[k];
            }
            w.rank[p] = rank;
            if (p == end - 1) w.total[1] = end - before - is;   // free pages below the end: as many as there are moves
        }
    }
}

// The others: counts by chunks, then ranks and lists.
__global__ __launch_bounds__(256) void pages_compact_count_kernel(ebrl_kv8_pool c, PgCompact w)
{
    __shared__ int red[4];
    const int used = pg_scan<4>(__popc(pg_used16(c, blockIdx.x * PG_CHUNK + threadIdx.x * 16)), red).y;
    if (threadIdx.x == 0) w.count[blockIdx.x] = used;
}
__global__ __launch_bounds__(256) void pages_compact_list_kernel(ebrl_kv8_pool c, int* used, PgCompact w)
{
    __shared__ int red[4];
    const int p = blockIdx.x * PG_CHUNK + threadIdx.x * 16;
    const unsigned m = pg_used16(c, p);
    const int2 u = pg_prefix(w.count, blockIdx.x, w.chunks, red);
    const int end = u.y;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        w.total[0] = end;
        if (end == 0) w.total[1] = 0;
        *used = end;
    }
    pg_place16(c, w, p, m, u.x + pg_scan<4>(__popc(m), red).x, end);
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
    // pieces of the moves, layer after layer
    const int groups = gridDim.x - table_groups, per_layer = moves * pieces;
    if (moves == 0) return;
    int u = blockIdx.x - table_groups, layer = u / per_layer;
    for (u -= layer * per_layer; layer < c.layers;) {
        const int k = u / pieces;
        pg_copy<true>(c, w.mover[moves - 1 - k], w.hole[k], layer, u - k * pieces, bytes);
        u += groups;
        if (u >= per_layer) {
            layer += u / per_layer;
            u %= per_layer;
        }
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
    return pg_chunks(c) + 3 * n + n * pages + 2 + std::min<int64_t>(n * pages, c->num_blocks);
}
static int64_t pg_compact_words(const ebrl_kv8_pool* c) {
    return pg_chunks(c) + c->num_blocks + 3 * ((int64_t)c->num_blocks / 2 + 1) + 2;
}
static bool pg_compact_ok(const ebrl_kv8_pool* c) {
    return pg_shape_ok(c) && (int64_t)(c->num_blocks / 2) * pg_pieces(c) <= (1 << 30);      // (16 TB a layer)
}
static int pg_status() { return hipGetLastError() == hipSuccess ? EBRL_OK : EBRL_E_HIP; }

// Layers that a workgroup of a reservation copies in: several where there are many, since what
// it looks up serves them all.
static int pg_reserve_step(const ebrl_kv8_pool* c, int32_t n) {
    return (int)std::max<int64_t>(1, std::min<int64_t>(8, (int64_t)n * pg_pieces(c) * c->layers / 2048));
}
static bool pg_reserve_ok(const ebrl_kv8_pool* c, int32_t n, int32_t max_count) {
    if (!pg_shape_ok(c) || n < 0 || n > PG_MAX_ROWS || max_count < 0 || n * pg_most_pages(c, max_count) > (1 << 30)) return false;
    const int step = pg_reserve_step(c, n);
    return (int64_t)n * pg_pieces(c) * ((c->layers + step - 1) / step) <= PG_MAX_GROUPS;
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
    if (!pg_reserve_ok(pool, n, max_count) || !pg_pool_ok(pool) || !lacking || (uintptr_t)lacking % 4) return EBRL_E_INVALID;
    const int64_t pages = pg_most_pages(pool, max_count);
    const int pieces = pg_pieces(pool);
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
    w.before = w.need + n;
    w.copy = w.before + n;
    w.total = w.copy + n;
    w.rank = w.total + 2;
    w.list = w.rank + (int64_t)n * pages;
    if (n <= PG_SMALL_ROWS && pool->num_blocks <= PG_SMALL_POOL && n * pages <= PG_SMALL_ENTRIES) {
        hipLaunchKernelGGL(pages_reserve_small_kernel, dim3(1), dim3(1024), 0, s, *pool, seq, pos0, count, max_count, lacking, w);
    } else {
        hipLaunchKernelGGL(pages_reserve_count_kernel, dim3(w.chunks + n), dim3(256), 0, s, *pool, seq, pos0, count, max_count, w);
        hipLaunchKernelGGL(pages_reserve_list_kernel, dim3(w.chunks + 1), dim3(256), 0, s, *pool, lacking, w);
    }
    if (n > 0) {
        const int step = pg_reserve_step(pool, n);
        hipLaunchKernelGGL(pages_reserve_kernel, dim3((unsigned)n * pieces, (pool->layers + step - 1) / step), dim3(256), 0, s,
                           *pool, seq, pos0, (int)pg_bytes(pool), pieces, step, w);
    }
    return pg_status();
}

int64_t ebrl_op_kv8_compact_workspace(const ebrl_kv8_pool* pool) {
    return pg_compact_ok(pool) ? pg_compact_words(pool) * 4 : EBRL_E_INVALID;
}

int ebrl_op_kv8_compact(const ebrl_kv8_pool* pool, int32_t* new_table, int32_t* new_refs, int32_t* used,
                        void* workspace, int64_t workspace_bytes, void* stream) {
    if (!pg_compact_ok(pool) || !pg_pool_ok(pool) || !new_table || !new_refs || !used ||
        ((uintptr_t)new_table | (uintptr_t)new_refs | (uintptr_t)used) % 4)
        return EBRL_E_INVALID;
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
    const int64_t most = (int64_t)(pool->num_blocks / 2) * pieces;
    const int copy_groups = (int)std::min<int64_t>(2048, most * pool->layers);
    if (pool->num_blocks <= PG_SMALL_POOL) {
        hipLaunchKernelGGL(pages_compact_small_kernel, dim3(1), dim3(1024), 0, s, *pool, used, w);
    } else {
        hipLaunchKernelGGL(pages_compact_count_kernel, dim3(w.chunks), dim3(256), 0, s, *pool, w);
        hipLaunchKernelGGL(pages_compact_list_kernel, dim3(w.chunks), dim3(256), 0, s, *pool, used, w);
    }
    hipLaunchKernelGGL(pages_compact_kernel, dim3(table_groups + copy_groups), dim3(256), 0, s, *pool, new_table,
                       new_refs, (int)pg_bytes(pool), pieces, table_groups, w);
    return pg_status();
}

}  // extern "C"
