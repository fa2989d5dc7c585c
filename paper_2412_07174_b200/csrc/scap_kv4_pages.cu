// Pages of the key / value cache: copy, fork, free, reserve, compact.
//
// The book-keeping (table, lengths, reference counts) lives on the device, so a decoding loop with beams runs in a graph without
// a look from the host.  Each call is one or two kernels: a plan by one CTA - whole numbers, a prefix sum over the sequences and one
// over the reference counts - and the copies of whole pages by all SMs, bound by memory.
//
// Which page goes to whom does not depend on timing: the lowest free pages are given out in the order of the request list.
#include "scap_kv4.cuh"

namespace scap {

constexpr int PG_THREADS = 1024;
constexpr int PG_COPY_THREADS = 256;
constexpr int PG_CHUNK = 32 * 1024;  // bytes a CTA copies at a time

struct PgCache {
    unsigned char *pages;
    long long stride;
    int n_pages, page_tokens, table_stride, n_seqs;
    int *table, *lens, *refs;
};

struct PgShared {
    int warp[32];
    int total;
};

// Exclusive prefix sum over the block; `total` is the sum.  All threads take part.
__device__ __forceinline__ int pg_scan(int v, PgShared &s, int &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int incl = v;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int up = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += up;
    }
    __syncthreads();
    if (lane == 31) s.warp[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        int w = s.warp[lane];
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int up = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += up;
        }
        s.warp[lane] = w;
        if (lane == 31) s.total = w;
    }
    __syncthreads();
    total = s.total;
    return incl - v + (warp > 0 ? s.warp[warp - 1] : 0);
}

__device__ __forceinline__ int pg_pages(const PgCache &c, int tokens) {  // pages of so many tokens, as far as a row of the table has room
    return tokens <= 0 ? 0 : (int)min((long long)c.table_stride, ((long long)tokens + c.page_tokens - 1) / c.page_tokens);
}
__device__ __forceinline__ bool pg_valid(const PgCache &c, int page) { return page >= 0 && page < c.n_pages; }

// Sixteen reference counts from page p on, as bits: which pages are held, which are free.
constexpr int PG_LOOK = 16;
__device__ __forceinline__ void pg_look(const PgCache &c, int p, uint32_t &held, uint32_t &free) {
    held = free = 0;
    if (p + PG_LOOK <= c.n_pages) {
        int r[PG_LOOK];
#pragma unroll
        for (int k = 0; k < PG_LOOK; k += 4) *reinterpret_cast<int4 *>(r + k) = __ldcg(reinterpret_cast<const int4 *>(c.refs + p + k));
#pragma unroll
        for (int k = 0; k < PG_LOOK; ++k) {
            held |= r[k] > 0 ? 1u << k : 0u;
            free |= r[k] == 0 ? 1u << k : 0u;
        }
    } else {
        for (int k = 0; p + k < c.n_pages; ++k) {
            const int r = __ldcg(c.refs + p + k);
            held |= r > 0 ? 1u << k : 0u;
            free |= r == 0 ? 1u << k : 0u;
        }
    }
}

// The lowest `want` free pages, in order, into list[0 ..]; returns how many there are.
__device__ __forceinline__ int pg_free_pages(const PgCache &c, int want, int *list, PgShared &s) {
    int found = 0;
    for (long long p0 = 0; p0 < c.n_pages && found < want; p0 += PG_LOOK * PG_THREADS) {
        const long long p = p0 + PG_LOOK * (int)threadIdx.x;
        uint32_t held = 0, free = 0;
        if (p < c.n_pages) pg_look(c, (int)p, held, free);
        int total, at = found + pg_scan(__popc(free), s, total);
        for (; free && at < want; free &= free - 1, ++at) list[at] = (int)p + __ffs(free) - 1;
        found += total;
    }
    __syncthreads();
    return min(found, want);
}

// ---- copies ------------------------------------------------------------------------------------------------------------------------------

// pages[dst[i]] = pages[src[i]]; a pair with a number that is no page is left out.  *count pairs, or `most` where there is no count.
// With place (compaction) the tables follow: a page at or behind *used has moved to place[page].
__global__ void __launch_bounds__(PG_COPY_THREADS) kv4_copy_kernel(const PgCache c, const int *src, const int *dst, const int *count, int most, const int *used, const int *place) {
    griddep_wait();
    griddep_launch_dependents();
    const int n = count ? min(__ldcg(count), most) : most;
    const long long per = (c.stride + PG_CHUNK - 1) / PG_CHUNK, all = per * n;
    for (long long w = blockIdx.x; w < all; w += gridDim.x) {
        const int i = (int)(w / per);
        const int from = __ldcg(src + i), to = __ldcg(dst + i);
        if (!pg_valid(c, from) || !pg_valid(c, to)) continue;
        const long long at = (w - i * per) * PG_CHUNK;
        const uint4 *a = reinterpret_cast<const uint4 *>(c.pages + from * c.stride + at);
        uint4 *b = reinterpret_cast<uint4 *>(c.pages + to * c.stride + at);
        const int words = (int)(min((long long)PG_CHUNK, c.stride - at) / 16);
        constexpr int U = PG_CHUNK / 16 / PG_COPY_THREADS;
        uint4 v[U];
        if (words == PG_CHUNK / 16) {
#pragma unroll
            for (int k = 0; k < U; ++k) v[k] = __ldcs(a + k * PG_COPY_THREADS + threadIdx.x);
#pragma unroll
            for (int k = 0; k < U; ++k) __stcs(b + k * PG_COPY_THREADS + threadIdx.x, v[k]);
        } else {
            for (int k = threadIdx.x; k < words; k += PG_COPY_THREADS) __stcs(b + k, __ldcs(a + k));
        }
    }
    if (place) {
        const long long cells = (long long)c.n_seqs * c.table_stride;
        const int first = __ldcg(used);
        for (long long i = (long long)blockIdx.x * PG_COPY_THREADS + threadIdx.x; i < cells; i += (long long)gridDim.x * PG_COPY_THREADS) {
            const int b = (int)(i / c.table_stride), t = (int)(i - (long long)b * c.table_stride);
            const int page = __ldcg(c.table + i);
            if (page >= first && page < c.n_pages && t < pg_pages(c, __ldcg(c.lens + b))) c.table[i] = __ldcg(place + page);
        }
    }
}

// ---- fork --------------------------------------------------------------------------------------------------------------------------------

// Request i: row dst[i] becomes a copy of row src[i].  Pages that are full are shared, the last and partial one gets a page of its own;
// from / to / count: the copies that are left to do.
__global__ void __launch_bounds__(PG_THREADS) kv4_fork_kernel(const PgCache c, const int *src, const int *dst, int n, int *fail, int *from, int *to, int *count, int *list) {
    __shared__ PgShared s;
    __shared__ int s_owner[SCAP_MAX_SEQS];  // first request that names a row as its destination
    __shared__ int s_src[PG_THREADS], s_dst[PG_THREADS], s_len[PG_THREADS], s_rank[PG_THREADS];
    constexpr int NOBODY = 0x7fffffff;
    griddep_wait();
    auto row_ok = [&](int b) { return b >= 0 && b < c.n_seqs; };
    for (int b = threadIdx.x; b < c.n_seqs; b += PG_THREADS) s_owner[b] = NOBODY;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += PG_THREADS) {
        const int b = __ldcg(dst + i);
        if (row_ok(b)) atomicMin(&s_owner[b], i);
    }
    __syncthreads();
    // This thread's request of a block of 1024: its rows and length into shared memory, and what it is - 0: left out, 1: shares all
    // pages, 2: needs one of its own.  (A destination's length changes only after its own request has been looked at for the last time.)
    auto look = [&](int i) {
        int what = 1;
        if (i < n) {
            const int a = __ldcg(src + i), b = __ldcg(dst + i);
            what = 0;
            if (row_ok(a) && row_ok(b) && s_owner[b] == i && s_owner[a] == NOBODY) {
                const int len = __ldcg(c.lens + a), there = __ldcg(c.lens + b);
                if (there <= 0 && (long long)len <= (long long)c.table_stride * c.page_tokens) what = len > 0 && len % c.page_tokens != 0 ? 2 : 1;
                s_len[threadIdx.x] = max(0, len);
            }
            s_src[threadIdx.x] = a;
            s_dst[threadIdx.x] = b;
        }
        return what;
    };
    int want = 0, what = 1;
    for (int i0 = 0; i0 < n; i0 += PG_THREADS) {
        what = look(i0 + (int)threadIdx.x);
        want += __syncthreads_count(what == 2);
    }
    const int have = pg_free_pages(c, want, list, s);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int before = 0, failed = 0;
    for (int i0 = 0; i0 < n; i0 += PG_THREADS) {
        if (n > PG_THREADS) what = look(i0 + (int)threadIdx.x);  // (else it is as it was)
        int total;
        const int rank = before + pg_scan(what == 2 ? 1 : 0, s, total);
        before += total;
        const bool lost = what == 2 && rank >= have;  // no page was left: the row stays empty
        s_rank[threadIdx.x] = what == 0 || lost ? -2 : (what == 2 ? rank : -1);
        failed += __syncthreads_count(what == 0 || lost);
        // rows, a warp per request, two at a time
        for (int k0 = warp; k0 < PG_THREADS && i0 + k0 < n; k0 += 2 * (PG_THREADS / 32)) {
            for (int t = lane; t < c.table_stride; t += 32) {
                int page[2];
                bool on[2];
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const int k = k0 + m * (PG_THREADS / 32);
                    on[m] = k < PG_THREADS && i0 + k < n && s_rank[k] != -2;
                    const int full = on[m] ? s_len[k] / c.page_tokens : -1;
                    page[m] = t < full || (t == full && s_rank[k] >= 0) ? __ldcg(c.table + (long long)s_src[k] * c.table_stride + t) : -1;
                }
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const int k = k0 + m * (PG_THREADS / 32);
                    if (!on[m]) continue;
                    const int r = s_rank[k];
                    if (t == s_len[k] / c.page_tokens && r >= 0) {  // the partial page
                        const int fresh = list[r];
                        from[r] = page[m];
                        to[r] = fresh;
                        c.refs[fresh] = 1;
                        page[m] = fresh;
                    } else if (pg_valid(c, page[m])) {
                        atomicAdd(c.refs + page[m], 1);
                    }
                    c.table[(long long)s_dst[k] * c.table_stride + t] = page[m];
                    if (t == 0) c.lens[s_dst[k]] = s_len[k];
                }
            }
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        *count = min(before, have);
        if (fail) *fail = failed;
    }
}

// ---- free --------------------------------------------------------------------------------------------------------------------------------

// A warp per row.  The row's length is taken and cleared in one step, so a row that is named twice is freed once.
__global__ void __launch_bounds__(PG_COPY_THREADS) kv4_free_kernel(const PgCache c, const int *rows, int n) {
    griddep_wait();
    griddep_launch_dependents();
    const int lane = threadIdx.x & 31, i = (int)((blockIdx.x * PG_COPY_THREADS + threadIdx.x) >> 5);
    if (i >= n) return;
    const int b = __ldcg(rows + i);
    if (b < 0 || b >= c.n_seqs) return;
    int len = 0;
    if (lane == 0) len = atomicExch(c.lens + b, 0);
    const int held = pg_pages(c, __shfl_sync(0xffffffffu, len, 0));
    if (held == 0) return;
    for (int t = lane; t < c.table_stride; t += 32) {
        int *at = c.table + (long long)b * c.table_stride + t;
        const int page = __ldcg(at);
        if (t < held && pg_valid(c, page)) atomicSub(c.refs + page, 1);
        *at = -1;
    }
}

// ---- reserve -----------------------------------------------------------------------------------------------------------------------------

// Room for add[b] more tokens of every sequence b, in their order.
__global__ void __launch_bounds__(PG_THREADS) kv4_reserve_kernel(const PgCache c, const int *add, int *fail, int *list) {
    __shared__ PgShared s;
    griddep_wait();
    // pages that sequence b asks for (one more than there are stands for any larger number): -1 where its table has no room for them
    auto more = [&](int b) {
        const long long len = max(0, __ldcg(c.lens + b)), sum = len + max(0, __ldcg(add + b));
        if (sum > (long long)c.table_stride * c.page_tokens || sum > 0x7fffffffll) return -1;
        return min(pg_pages(c, (int)sum) - pg_pages(c, (int)len), c.n_pages + 1);
    };
    long long want = 0;
    int m = 0, first_of = 0;
    for (int b0 = 0; b0 < c.n_seqs; b0 += PG_THREADS) {
        const int b = b0 + (int)threadIdx.x;
        int total;
        m = b < c.n_seqs ? more(b) : 0;
        first_of = pg_scan(max(0, m), s, total);
        want += total;
    }
    const int have = pg_free_pages(c, (int)min(want, (long long)c.n_pages), list, s);
    long long before = 0;
    int failed = 0, first_before = 0;  // pages asked for by the blocks of sequences before, and by the last of these
    for (int b0 = 0; b0 < c.n_seqs; b0 += PG_THREADS) {
        const int b = b0 + (int)threadIdx.x;
        if (c.n_seqs > PG_THREADS) {  // (else all is as it was)
            int total;
            m = b < c.n_seqs ? more(b) : 0;
            first_of = pg_scan(max(0, m), s, total);
            __syncthreads();
            before += first_before;
            first_before = total;
        }
        const long long first = before + first_of;
        const bool ok = m == 0 || (m > 0 && first + m <= have);
        if (b < c.n_seqs && ok) {
            const int len = max(0, __ldcg(c.lens + b)), held = pg_pages(c, len);
            for (int k = 0; k < m; ++k) {
                const int page = list[first + k];
                c.table[(long long)b * c.table_stride + held + k] = page;
                c.refs[page] = 1;
            }
            c.lens[b] = len + max(0, __ldcg(add + b));
        }
        failed += __syncthreads_count(b < c.n_seqs && !ok);
    }
    if (threadIdx.x == 0 && fail) *fail = failed;
}

// ---- compact -----------------------------------------------------------------------------------------------------------------------------

// The used pages at or behind number `used` (that of all used pages) move, in order, into the free ones before it: sources and
// destinations have nothing in common, so all copies go side by side.  place[p] = where page p went, for those that move.
__global__ void __launch_bounds__(PG_THREADS) kv4_compact_kernel(const PgCache c, int *used_out, int *from, int *to, int *count, int *place) {
    __shared__ PgShared s;
    griddep_wait();
    int used = 0;
    for (long long p0 = 0; p0 < c.n_pages; p0 += PG_LOOK * PG_THREADS) {
        const long long p = p0 + PG_LOOK * (int)threadIdx.x;
        uint32_t held = 0, free = 0;
        if (p < c.n_pages) pg_look(c, (int)p, held, free);
        int total;
        pg_scan(__popc(held), s, total);
        used += total;
    }
    int holes = 0, moving = 0;
    for (long long p0 = 0; p0 < c.n_pages; p0 += PG_LOOK * PG_THREADS) {
        const long long p = p0 + PG_LOOK * (int)threadIdx.x;
        uint32_t held = 0, free = 0;
        if (p < c.n_pages) pg_look(c, (int)p, held, free);
        // bits of the pages before `used`
        const uint32_t low = p + PG_LOOK <= used ? 0xffffu : (p >= used ? 0u : (1u << (used - (int)p)) - 1u);
        uint32_t hole = ~held & low, move = held & ~low;
        // both sums in one scan: a round has 2^14 pages
        int total;
        const int at = pg_scan(__popc(hole) | (__popc(move) << 16), s, total);
        int h = holes + (at & 0xffff), m = moving + (at >> 16);
        for (; hole; hole &= hole - 1) to[h++] = (int)p + __ffs(hole) - 1;
        for (; move; move &= move - 1) from[m++] = (int)p + __ffs(move) - 1;
        holes += total & 0xffff;
        moving += total >> 16;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < moving; i += PG_THREADS) {  // as many holes as movers
        const int a = from[i], b = to[i];
        place[a] = b;
        c.refs[b] = c.refs[a];
        c.refs[a] = 0;
    }
    if (threadIdx.x == 0) {
        *count = moving;
        *used_out = used;
    }
}

// ---- host --------------------------------------------------------------------------------------------------------------------------------

static bool aligned4(const int *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }  // (one number: any int will do)

static scap_status pg_check(const scap_kv4 *c, bool rows) {
    if (!c || !c->pages) return SCAP_ERR_INVALID_ARG;
    if (rows && (!c->table || !c->lens || !c->refs)) return SCAP_ERR_INVALID_ARG;
    if (c->n_pages < 1 || c->page_stride < 16 || c->page_stride > ((size_t)1 << 40)) return SCAP_ERR_SHAPE;
    if (rows && (c->page_tokens < KV_TILE || c->page_tokens > 4096 || c->page_tokens % KV_TILE || c->table_stride < 1 || c->n_seqs < 1 || c->n_seqs > SCAP_MAX_SEQS ||
                 c->n_pages > SCAP_MAX_PAGES))
        return SCAP_ERR_SHAPE;
    if (!aligned16(c->pages) || c->page_stride % 16 || (rows && (!aligned16(c->table) || !aligned16(c->lens) || !aligned16(c->refs)))) return SCAP_ERR_ALIGN;
    return SCAP_OK;
}

static PgCache pg_cache(const scap_kv4 *c) {
    PgCache p;
    p.pages = reinterpret_cast<unsigned char *>(c->pages);
    p.stride = (long long)c->page_stride;
    p.n_pages = c->n_pages; p.page_tokens = c->page_tokens; p.table_stride = c->table_stride; p.n_seqs = c->n_seqs;
    p.table = c->table; p.lens = c->lens; p.refs = c->refs;
    return p;
}

// Workspace: counters, then three lists of as many entries as there are pages or requests.
struct PgSpace {
    int *count, *used, *from, *to, *list;
};
static size_t pg_list(int n_pages, int n) { return align_up((size_t)(n_pages > n ? n_pages : n) * sizeof(int), 16); }
static PgSpace pg_space(void *ws, int n_pages, int n) {
    unsigned char *p = reinterpret_cast<unsigned char *>(ws);
    const size_t list = pg_list(n_pages, n);
    PgSpace s;
    s.count = reinterpret_cast<int *>(p);
    s.used = s.count + 1;
    s.from = reinterpret_cast<int *>(p + 16);
    s.to = reinterpret_cast<int *>(p + 16 + list);
    s.list = reinterpret_cast<int *>(p + 16 + 2 * list);
    return s;
}

static cudaError_t pg_copy(const PgCache &c, const int *src, const int *dst, const int *count, int most, cudaStream_t st, const int *used = nullptr, const int *place = nullptr) {
    const long long work = (c.stride + PG_CHUNK - 1) / PG_CHUNK * (long long)most, cap = 8LL * sm_count();
    return launch(kv4_copy_kernel, dim3((unsigned)(work < cap ? work : cap)), dim3(PG_COPY_THREADS), 0, st, g_tune.pdl != 0, c, src, dst, count, most, used, place);
}

}  // namespace scap

using namespace scap;

extern "C" size_t scap_kv4_pages_workspace(int n_pages, int n) {
    if (n_pages < 1 || n_pages > SCAP_MAX_PAGES || n < 1 || n > SCAP_MAX_SEQS) return 0;
    return 16 + 3 * pg_list(n_pages, n);
}

extern "C" scap_status scap_kv4_copy(const scap_kv4 *cache, const int *src, const int *dst, int n, scap_stream_t stream) {
    scap_status s = pg_check(cache, false);
    if (s != SCAP_OK) return s;
    if (n < 0 || n > SCAP_MAX_PAGES) return SCAP_ERR_SHAPE;
    if (n == 0) return SCAP_OK;
    if (!src || !dst) return SCAP_ERR_INVALID_ARG;
    if (!aligned16(src) || !aligned16(dst)) return SCAP_ERR_ALIGN;
    s = check_device();
    if (s != SCAP_OK) return s;
    return cuda_status(pg_copy(pg_cache(cache), src, dst, nullptr, n, reinterpret_cast<cudaStream_t>(stream)));
}

extern "C" scap_status scap_kv4_fork(const scap_kv4 *cache, const int *src, const int *dst, int n, int *fail_out, void *ws, size_t ws_bytes, scap_stream_t stream) {
    scap_status s = pg_check(cache, true);
    if (s != SCAP_OK) return s;
    if (n < 0 || n > cache->n_seqs) return SCAP_ERR_SHAPE;
    if (n == 0) return SCAP_OK;
    if (!src || !dst || !ws) return SCAP_ERR_INVALID_ARG;
    if (!aligned16(src) || !aligned16(dst) || !aligned16(ws) || !aligned4(fail_out)) return SCAP_ERR_ALIGN;
    if (ws_bytes < scap_kv4_pages_workspace(cache->n_pages, n)) return SCAP_ERR_WORKSPACE;
    s = check_device();
    if (s != SCAP_OK) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const PgCache c = pg_cache(cache);
    const PgSpace w = pg_space(ws, cache->n_pages, n);
    cudaError_t e = launch(kv4_fork_kernel, dim3(1), dim3(PG_THREADS), 0, st, g_tune.pdl != 0, c, src, dst, n, fail_out, w.from, w.to, w.count, w.list);
    if (e != cudaSuccess) return cuda_status(e);
    return cuda_status(pg_copy(c, w.from, w.to, w.count, n, st));
}

extern "C" scap_status scap_kv4_free(const scap_kv4 *cache, const int *rows, int n, scap_stream_t stream) {
    scap_status s = pg_check(cache, true);
    if (s != SCAP_OK) return s;
    if (n < 0 || n > SCAP_MAX_SEQS) return SCAP_ERR_SHAPE;
    if (n == 0) return SCAP_OK;
    if (!rows) return SCAP_ERR_INVALID_ARG;
    if (!aligned16(rows)) return SCAP_ERR_ALIGN;
    s = check_device();
    if (s != SCAP_OK) return s;
    const int per = PG_COPY_THREADS / 32;
    return cuda_status(launch(kv4_free_kernel, dim3((n + per - 1) / per), dim3(PG_COPY_THREADS), 0, reinterpret_cast<cudaStream_t>(stream), g_tune.pdl != 0, pg_cache(cache), rows, n));
}

extern "C" scap_status scap_kv4_reserve(const scap_kv4 *cache, const int *add, int *fail_out, void *ws, size_t ws_bytes, scap_stream_t stream) {
    scap_status s = pg_check(cache, true);
    if (s != SCAP_OK) return s;
    if (!add || !ws) return SCAP_ERR_INVALID_ARG;
    if (!aligned16(add) || !aligned16(ws) || !aligned4(fail_out)) return SCAP_ERR_ALIGN;
    if (ws_bytes < scap_kv4_pages_workspace(cache->n_pages, 1)) return SCAP_ERR_WORKSPACE;
    s = check_device();
    if (s != SCAP_OK) return s;
    const PgSpace w = pg_space(ws, cache->n_pages, 1);
    return cuda_status(launch(kv4_reserve_kernel, dim3(1), dim3(PG_THREADS), 0, reinterpret_cast<cudaStream_t>(stream), g_tune.pdl != 0, pg_cache(cache), add, fail_out, w.list));
}

extern "C" scap_status scap_kv4_compact(const scap_kv4 *cache, int *used_out, void *ws, size_t ws_bytes, scap_stream_t stream) {
    scap_status s = pg_check(cache, true);
    if (s != SCAP_OK) return s;
    if (!ws) return SCAP_ERR_INVALID_ARG;
    if (!aligned16(ws) || !aligned4(used_out)) return SCAP_ERR_ALIGN;
    if (ws_bytes < scap_kv4_pages_workspace(cache->n_pages, 1)) return SCAP_ERR_WORKSPACE;
    s = check_device();
    if (s != SCAP_OK) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const PgCache c = pg_cache(cache);
    const PgSpace w = pg_space(ws, cache->n_pages, 1);
    int *used = used_out ? used_out : w.used;
    cudaError_t e = launch(kv4_compact_kernel, dim3(1), dim3(PG_THREADS), 0, st, g_tune.pdl != 0, c, used, w.from, w.to, w.count, w.list);
    if (e != cudaSuccess) return cuda_status(e);
    return cuda_status(pg_copy(c, w.from, w.to, w.count, cache->n_pages, st, used, w.list));
}
