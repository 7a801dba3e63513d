// The pages of a paged cache: who holds them, handing out, sharing, taking back
// and moving them.
//
// The state is the requests' block tables and lengths and, for each page, the
// number of table entries that name it (ref; 0: the page is free).  There is no
// free list: giving pages back is an atomic subtraction and sharing them an atomic
// addition, whose order does not matter, and the free pages are found by counting
// zeros of ref, 4 bytes a page, in parallel and in the order of their ids.  So every
// result is a function of the inputs, and pages are handed out lowest ids first,
// which keeps the pool dense.  (A list of free pages would save that reading, 1 MB
// for 2^18 pages, and its order would depend on the atomics'.)
//
// What one launch writes another workgroup reads in the next launch only (a
// device-scope fence would write back the whole L2 of an XCD).  The integers are
// bound by launches and by their few dependent loads, the copies by HBM.
#include <algorithm>

#include "device_common.h"
#include "kernels.h"

namespace dspark {

namespace {

constexpr int kPgThreads = 1024;
constexpr int kPgWaves = kPgThreads / DSPARK_WAVE;
constexpr int kPgChunk = kPgThreads;    // pages that a workgroup counts
constexpr int kPgRequests = 8192;       // at most (checked by the caller)
constexpr int kPgRounds = kPgRequests / kPgThreads;
constexpr int kRowThreads = 256;        // of a request's pages
constexpr int kCopyThreads = 256;
constexpr int kCopyUnit = kCopyThreads * 16 * 4;  // bytes of a page that a workgroup copies at a time
constexpr int kCopyGrid = 512;
constexpr int kSmallBytes = 512;        // of a page in a small buffer, at most
constexpr int kSmallThreads = 16;       // that copy it
constexpr int kCopyBufs = 64;           // buffers of a launch

// Workspace, in int32 words (256-byte pieces)
struct PgLayout {
    size_t head, count, upto, col, copies, last, grown, src, dst, owner, owners, bytes;
};
__host__ __device__ inline int pg_chunks(int num_pages) { return (num_pages + kPgChunk - 1) / kPgChunk; }
PgLayout pg_layout(int R, int N) {
    auto up = [](size_t n) { return (n * 4 + 255) / 256 * 64; };
    PgLayout l;
    l.head = 0;
    l.count = 64;                     // free pages of each chunk
    l.upto = l.count + up(pg_chunks(N));
    l.col = l.upto + up(R);           // reserve: per request; fork: length of each pair
    l.copies = l.col + up(R);
    l.last = l.copies + up(R);
    l.grown = l.last + up(R);
    l.src = l.grown + up(R);          // pages to copy, from
    l.dst = l.src + up(std::max(R, N));  // and to
    l.owner = l.dst + up(std::max(R, N));
    l.owners = l.owner + up(std::max(R, N));
    l.bytes = (l.owners + up(N)) * 4;
    return l;
}

struct PgParams {
    PageArgs a;
    int32_t* head;   // [0] pages to copy, [1] pages in use
    int32_t* count;
    int32_t* upto;    // [R] pages that the requests up to r need
    int32_t* col;     // [R] first table entry to write, and flags
    int32_t* copies;  // [R] copies of the requests up to r
    int32_t* last;    // [R] the partial page
    int32_t* grown;   // [R] tokens afterwards
    int32_t* src;
    int32_t* dst;
    int32_t* owner;
    int32_t* owners;
};
PgParams pg_params(const PageArgs& a, void* ws) {
    const PgLayout l = pg_layout(a.R, a.num_pages);
    int32_t* w = (int32_t*)ws;
    return PgParams{a,          w + l.head,  w + l.count, w + l.upto, w + l.col,   w + l.copies,
                    w + l.last, w + l.grown, w + l.src,   w + l.dst,  w + l.owner, w + l.owners};
}

// Words that several threads of a workgroup exchange through memory: device-scope
// accesses, which bypass the caches that a plain load might find stale.
__device__ __forceinline__ void put(int32_t* p, int v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ int get(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// this thread's accesses are done, and then everyone's
__device__ __forceinline__ void exchange_barrier() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

template <typename T>
__device__ __forceinline__ T wave_incl(T v) {
    const int lane = threadIdx.x & (DSPARK_WAVE - 1);
#pragma unroll
    for (int o = 1; o < DSPARK_WAVE; o <<= 1) {
        const T t = __shfl_up(v, o, DSPARK_WAVE);
        if (lane >= o) v += t;
    }
    return v;
}
__device__ __forceinline__ int wave_total(int v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, DSPARK_WAVE);
    return v;
}

// Sums over a workgroup of kPgThreads.  `s`: kPgWaves words of its own for each call.
__device__ __forceinline__ int group_total(int v, int* s) {
    v = wave_total(v);
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    int t = 0;
#pragma unroll
    for (int w = 0; w < kPgWaves; ++w) t += s[w];
    return t;
}
// inclusive prefix sum; `all` gets the total
template <typename T>
__device__ __forceinline__ T group_incl(T v, T* s, T& all) {
    const T incl = wave_incl(v);
    if ((threadIdx.x & 63) == 63) s[threadIdx.x >> 6] = incl;
    __syncthreads();
    T before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < kPgWaves; ++w) {
        before += w < (int)(threadIdx.x >> 6) ? s[w] : 0;
        all += s[w];
    }
    return incl + before;
}

__device__ __forceinline__ int pages_of(int tokens, int page) { return (tokens + page - 1) / page; }

// ---- free pages, counted by chunk

__device__ __forceinline__ bool is_free(const PageArgs& a, int p) { return p < a.num_pages && a.ref[p] == 0; }

__device__ void count_chunk(const PgParams& p, int chunk) {
    __shared__ int s[kPgWaves];
    const int n = group_total(is_free(p.a, chunk * kPgChunk + threadIdx.x), s);
    if (threadIdx.x == 0) p.count[chunk] = n;
}

// free pages before chunk `chunk`, and in all
__device__ __forceinline__ void free_before(const PgParams& p, int chunk, int& before, int& all, int* s) {
    int b = 0, t = 0;
    for (int i = threadIdx.x; i < pg_chunks(p.a.num_pages); i += kPgThreads) {
        const int n = p.count[i];
        t += n;
        if (i < chunk) b += n;
    }
    before = group_total(b, s);
    all = group_total(t, s + kPgWaves);
}

// ---- reserve

// What request r needs for its q_len more tokens.
struct Need {
    int pages;   // pages to hand out, without the copy's
    int shared;  // the last, partial page is held by others too
    int last;    // which it is
    int col;     // first table entry past it
    int grown;   // tokens afterwards; 0: the request's values are malformed
};
__device__ __forceinline__ Need need_of(const PageArgs& a, const int32_t* cu_q, int r) {
    const int kv = a.kv_len[r];
    const int64_t ql = (int64_t)cu_q[r + 1] - cu_q[r];
    if (kv < 0 || ql < 0 || kv + ql > (int64_t)a.max_pages * a.page) return Need{0, 0, 0, 0, 0};
    const int grown = kv + (int)ql, have = pages_of(kv, a.page);
    Need n{pages_of(grown, a.page) - have, 0, 0, have, grown};
    if (ql > 0 && kv % a.page) {
        n.last = a.block_table[(int64_t)r * a.max_pages + kv / a.page];
        if ((unsigned)n.last >= (unsigned)a.num_pages) return Need{0, 0, 0, 0, 0};
        n.shared = a.ref[n.last] > 1;
    }
    return n;
}

// Workgroup 0: what every request needs, added up in request order; the others count
// the free pages.  A shared partial page whose holders all grow stays with the last of
// them, the others copy it.
constexpr int kCopy = 1 << 30;                 // flags beside the first table entry: copies its partial page,
constexpr int kKeep = 1 << 29;                 // keeps one that others copy,
constexpr int kNone = 1 << 28;                 // needs nothing of anyone
constexpr int kColMask = kNone - 1;            // (max_pages is below 2^27)
__global__ __launch_bounds__(kPgThreads) void pg_plan(PgParams p, const int32_t* cu_q) {
    if (blockIdx.x > 0) {
        count_chunk(p, blockIdx.x - 1);
        return;
    }
    const PageArgs& a = p.a;
    __shared__ int64_t s_sum[kPgRounds][kPgWaves];
    __shared__ int s_copies[kPgRounds][kPgWaves];
    Need n[kPgRounds];
    bool any = false;
#pragma unroll
    for (int k = 0; k < kPgRounds; ++k) {
        const int r = k * kPgThreads + threadIdx.x;
        n[k] = r < a.R ? need_of(a, cu_q, r) : Need{0, 0, 0, 0, 0};
        if (n[k].shared) {
            any = true;
            put(&p.owner[n[k].last], -1);
            put(&p.owners[n[k].last], 0);
        }
    }
    if (__syncthreads_or(any)) {
        exchange_barrier();
#pragma unroll
        for (int k = 0; k < kPgRounds; ++k)
            if (n[k].shared) {
                atomicMax(&p.owner[n[k].last], k * kPgThreads + (int)threadIdx.x);
                atomicAdd(&p.owners[n[k].last], 1);
            }
        exchange_barrier();
    }
    int64_t needed = 0;  // by the rounds before
    int copied = 0;
#pragma unroll
    for (int k = 0; k < kPgRounds; ++k) {
        if (k * kPgThreads >= a.R) break;  // uniform
        const int r = k * kPgThreads + threadIdx.x;
        const bool keep = n[k].shared && get(&p.owners[n[k].last]) == a.ref[n[k].last] && get(&p.owner[n[k].last]) == r;
        const int copy = n[k].shared && !keep;
        int64_t all;
        int copies;
        const int64_t upto = needed + group_incl<int64_t>(n[k].pages + copy, s_sum[k], all);
        const int c = copied + group_incl<int>(copy, s_copies[k], copies);
        if (r < a.R) {
            // (beyond the number of pages a sum only has to stay there)
            p.upto[r] = (int)min(upto, (int64_t)0x7fffffff);
            p.copies[r] = c;
            p.col[r] = (n[k].col - copy) | (copy ? kCopy : 0) | (keep ? kKeep : 0) | (n[k].pages + copy == 0 && !keep ? kNone : 0);
            p.last[r] = n[k].last;
            p.grown[r] = n[k].grown;
        }
        needed += all;
        copied += copies;
    }
}

// Hands out the free pages, lowest ids first, to the requests in order, as far as they
// go: the free page of rank j goes to the request whose sum of needs passes j.  A request
// is served when what it and all before it need is there, or when it needs nothing; one
// that keeps a page needs the others' copies of it.
__global__ __launch_bounds__(kPgThreads) void pg_assign(PgParams p, int32_t* step_len) {
    const PageArgs& a = p.a;
    __shared__ int s_upto[kPgRequests];
    __shared__ int s_sum[6][kPgWaves];
    int before, free;
    free_before(p, blockIdx.x, before, free, s_sum[0]);
    // pages and copies of the requests that are served
    int given = 0, copies = 0;
    for (int r = threadIdx.x; r < a.R; r += kPgThreads) {
        const int u = p.upto[r];
        s_upto[r] = u;
        if (u <= free) {
            given = max(given, u);
            copies = max(copies, p.copies[r]);
        }
    }
    for (int o = 32; o > 0; o >>= 1) {
        given = max(given, __shfl_xor(given, o, DSPARK_WAVE));
        copies = max(copies, __shfl_xor(copies, o, DSPARK_WAVE));
    }
    if ((threadIdx.x & 63) == 0) s_sum[2][threadIdx.x >> 6] = given, s_sum[3][threadIdx.x >> 6] = copies;
    __syncthreads();
    for (int w = 0; w < kPgWaves; ++w) given = max(given, s_sum[2][w]), copies = max(copies, s_sum[3][w]);
    if (blockIdx.x == 0 && threadIdx.x == 0) p.head[0] = copies;

    if (before < given) {  // uniform
        const int page = blockIdx.x * kPgChunk + threadIdx.x;
        const bool mine = is_free(a, page);
        int all;
        const int rank = before + group_incl<int>(mine, s_sum[4], all) - 1;
        if (mine && rank < given) {
            int lo = 0, hi = a.R - 1;  // first request with upto > rank
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (s_upto[mid] > rank) hi = mid;
                else lo = mid + 1;
            }
            const int at = rank - (lo ? s_upto[lo - 1] : 0);
            const int c = p.col[lo];
            if ((c & kCopy) && at == 0) p.dst[p.copies[lo] - 1] = page;
            a.block_table[(int64_t)lo * a.max_pages + (c & kColMask) + at] = page;
            a.ref[page] = 1;
        }
    }
    for (int r = blockIdx.x * kPgThreads + threadIdx.x; r < a.R; r += gridDim.x * kPgThreads) {
        const int c = p.col[r];
        const bool served = s_upto[r] <= free || (c & kNone);
        step_len[r] = served ? p.grown[r] : 0;
        if (served && (c & kCopy)) {
            p.src[p.copies[r] - 1] = p.last[r];
            atomicSub(&a.ref[p.last[r]], 1);  // stays above 0: someone keeps the page
        }
    }
}

// ---- commit and trim: a workgroup per request gives back the pages past its new length

__global__ __launch_bounds__(kRowThreads) void pg_drop(PageArgs a, const int32_t* step_len, const int32_t* cu_q,
                                                       const int32_t* accepted, const int32_t* new_len) {
    const int r = blockIdx.x;
    const int64_t most = (int64_t)a.max_pages * a.page;
    int now, keep;
    if (cu_q) {
        now = step_len[r];
        const int64_t ql = (int64_t)cu_q[r + 1] - cu_q[r];
        if (now < 1 || now > most || ql < 0 || ql > now) return;
        const int64_t kept = accepted ? min(max((int64_t)accepted[r] + 1, (int64_t)0), ql) : ql;
        keep = now - (int)(ql - kept);
    } else {
        now = a.kv_len[r];
        if (now < 1 || now > most) return;
        keep = min(now, max(new_len[r], 0));
    }
    const int32_t* row = a.block_table + (int64_t)r * a.max_pages;
    const int end = pages_of(now, a.page);
    for (int i = pages_of(keep, a.page) + threadIdx.x; i < end; i += kRowThreads) {
        const int pg = row[i];
        if ((unsigned)pg < (unsigned)a.num_pages) atomicSub(&a.ref[pg], 1);
    }
    __syncthreads();  // everyone has read kv_len
    if (threadIdx.x == 0) a.kv_len[r] = keep;
}

// ---- fork

// Tokens that each pair's child gets (-1: the pair is skipped).  One workgroup.
__global__ __launch_bounds__(kPgThreads) void pg_fork_plan(PgParams p, const int32_t* parent, const int32_t* child,
                                                           const int32_t* len, int n) {
    const PageArgs& a = p.a;
    auto in = [&](int r) { return (unsigned)r < (unsigned)a.R; };
    for (int i = threadIdx.x; i < n; i += kPgThreads)
        if (in(child[i])) put(&p.owner[child[i]], 0x7fffffff);
    exchange_barrier();
    for (int i = threadIdx.x; i < n; i += kPgThreads)
        if (in(child[i])) atomicMin(&p.owner[child[i]], i);
    exchange_barrier();
    for (int i = threadIdx.x; i < n; i += kPgThreads) {
        const int from = parent[i], to = child[i];
        int tokens = -1;
        if (in(from) && in(to) && from != to && a.kv_len[to] == 0 && get(&p.owner[to]) == i) {
            const int kv = a.kv_len[from];
            if (kv >= 0 && kv <= (int64_t)a.max_pages * a.page) tokens = len ? min(kv, max(len[i], 0)) : kv;
        }
        p.col[i] = tokens;
    }
}

__global__ __launch_bounds__(kRowThreads) void pg_fork(PgParams p, const int32_t* parent, const int32_t* child) {
    const PageArgs& a = p.a;
    const int tokens = p.col[blockIdx.x];
    if (tokens < 0) return;
    const int from = parent[blockIdx.x], to = child[blockIdx.x];
    for (int i = threadIdx.x; i < pages_of(tokens, a.page); i += kRowThreads) {
        const int pg = a.block_table[(int64_t)from * a.max_pages + i];
        a.block_table[(int64_t)to * a.max_pages + i] = pg;
        if ((unsigned)pg < (unsigned)a.num_pages) atomicAdd(&a.ref[pg], 1);
    }
    if (threadIdx.x == 0) a.kv_len[to] = tokens;
}

// ---- compact

__global__ __launch_bounds__(kPgThreads) void pg_count(PgParams p) { count_chunk(p, blockIdx.x); }

// With n pages in use, the k-th used page from id n on goes to the k-th free page below
// n: dst[k] and src[k], and owner[page] = k for the pages that move (-1: stays).
__global__ __launch_bounds__(kPgThreads) void pg_rank(PgParams p, int32_t* used) {
    const PageArgs& a = p.a;
    __shared__ int s_sum[4][kPgWaves];
    int before, free;
    free_before(p, blockIdx.x, before, free, s_sum[0]);
    const int n = a.num_pages - free;
    const int page = blockIdx.x * kPgChunk + threadIdx.x;
    const bool open = is_free(a, page);
    // free pages below n: those of the chunks before n's, and of its own up to n
    const int nc = n / kPgChunk;
    int part = 0;
    for (int i = threadIdx.x; i < nc; i += kPgThreads) part += p.count[i];
    const int edge = nc * kPgChunk + (int)threadIdx.x;
    part += edge < n && is_free(a, edge);
    const int holes = group_total(part, s_sum[2]);
    int all;
    const int free_upto = before + group_incl<int>(open, s_sum[3], all);
    if (page < a.num_pages) {
        int k = -1;
        if (page < n) {
            if (open) p.dst[free_upto - 1] = page;
        } else if (!open) {
            k = page - free_upto - (n - holes);  // used pages in [n, page)
            p.src[k] = page;
        }
        p.owner[page] = k;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        p.head[0] = holes;
        p.head[1] = n;
        *used = n;
    }
}

// Tables and counts follow the moved pages.  Workgroups: requests, then pages.
__global__ __launch_bounds__(kRowThreads) void pg_follow(PgParams p) {
    const PageArgs& a = p.a;
    if ((int)blockIdx.x >= a.R) {
        const int k = ((int)blockIdx.x - a.R) * kRowThreads + (int)threadIdx.x;
        if (k < p.head[0]) {
            a.ref[p.dst[k]] = a.ref[p.src[k]];
            a.ref[p.src[k]] = 0;
        }
        return;
    }
    const int r = blockIdx.x, n = p.head[1], kv = a.kv_len[r];
    if (kv < 1 || kv > (int64_t)a.max_pages * a.page) return;
    int32_t* row = a.block_table + (int64_t)r * a.max_pages;
    for (int i = threadIdx.x; i < pages_of(kv, a.page); i += kRowThreads) {
        const int pg = row[i];
        if (pg < n || pg >= a.num_pages) continue;
        const int k = p.owner[pg];
        if (k >= 0) row[i] = p.dst[k];
    }
}

// ---- copies of whole pages, src[k] to dst[k]: workgroups walk (page, unit), a unit being
// kCopyUnit bytes of a large buffer's page or those of all small buffers together (the
// scales of a page are a few bytes: as units of their own they were a fifth of the walk).
// 2 GB there and back in 64 KB pieces: 392 us, 5.4 TB/s, as a large copy; 8% more with four
// times as many workgroups or with stores that stay in the caches, 20% with half as many.

struct CopyParams {
    const int32_t* pairs;
    const int32_t* src;
    const int32_t* dst;
    int n_large, n_small;
    int large;  // units of a page in the large buffers
    int units;  // in all
    struct {
        char* base;
        int64_t stride, bytes;
        int unit, wide;  // first unit; bytes of an access
    } b[kCopyBufs];      // large ones, then small ones
};

typedef uint32_t Chunk16 __attribute__((ext_vector_type(4)));

// (stores past the caches, whose lines the copy would not read again)
template <typename T, int Threads>
__device__ __forceinline__ void copy_unit(const char* from, char* to, int64_t bytes, int thread) {
    constexpr int kBatch = 4;
    const T* f = (const T*)from;
    T* t = (T*)to;
    const int n = (int)(bytes / (int64_t)sizeof(T));
    for (int i = thread; i < n; i += Threads * kBatch) {
        T v[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (i + k * Threads < n) v[k] = f[i + k * Threads];
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (i + k * Threads < n) __builtin_nontemporal_store(v[k], t + i + k * Threads);
    }
}

__global__ __launch_bounds__(kCopyThreads) void pg_copy(CopyParams p) {
    const int64_t work = (int64_t)*p.pairs * p.units;
    for (int64_t w = blockIdx.x; w < work; w += gridDim.x) {
        const int pair = (int)(w / p.units), u = (int)(w - (int64_t)pair * p.units);
        const int64_t src = p.src[pair], dst = p.dst[pair];
        if (u < p.large) {
            int b = 0;
            while (b + 1 < p.n_large && p.b[b + 1].unit <= u) ++b;
            const int64_t at = (int64_t)(u - p.b[b].unit) * kCopyUnit, n = min((int64_t)kCopyUnit, p.b[b].bytes - at);
            const char* from = p.b[b].base + src * p.b[b].stride + at;
            char* to = p.b[b].base + dst * p.b[b].stride + at;
            if (p.b[b].wide == 16) copy_unit<Chunk16, kCopyThreads>(from, to, n, threadIdx.x);
            else if (p.b[b].wide == 4) copy_unit<uint32_t, kCopyThreads>(from, to, n, threadIdx.x);
            else copy_unit<uint8_t, kCopyThreads>(from, to, n, threadIdx.x);
        } else {
            for (int i = threadIdx.x / kSmallThreads; i < p.n_small; i += kCopyThreads / kSmallThreads) {
                const auto& b = p.b[p.n_large + i];
                const char* from = b.base + src * b.stride;
                char* to = b.base + dst * b.stride;
                const int t = threadIdx.x % kSmallThreads;
                if (b.wide == 4) copy_unit<uint32_t, kSmallThreads>(from, to, b.bytes, t);
                else copy_unit<uint8_t, kSmallThreads>(from, to, b.bytes, t);
            }
        }
    }
}

hipError_t copy_pages(const PgParams& p, const PageBuffer* bufs, int n_bufs, hipStream_t s) {
    for (int at = 0; at < n_bufs; at += kCopyBufs) {
        CopyParams c;
        c.pairs = p.head;
        c.src = p.src;
        c.dst = p.dst;
        c.n_large = c.n_small = c.large = 0;
        const int n = std::min(kCopyBufs, n_bufs - at);
        for (int small = 0; small < 2; ++small)
            for (int i = 0; i < n; ++i) {
                const PageBuffer& b = bufs[at + i];
                if ((b.bytes <= kSmallBytes) != (small == 1)) continue;
                auto& to = c.b[c.n_large + c.n_small];
                const uint64_t all = (uint64_t)(uintptr_t)b.base | (uint64_t)b.stride | (uint64_t)b.bytes;
                to.base = (char*)b.base;
                to.stride = b.stride;
                to.bytes = b.bytes;
                to.unit = c.large;
                to.wide = !small && all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 1;
                if (small) {
                    ++c.n_small;
                } else {
                    ++c.n_large;
                    c.large += (int)((b.bytes + kCopyUnit - 1) / kCopyUnit);
                }
            }
        c.units = c.large + (c.n_small > 0);
        hipLaunchKernelGGL(pg_copy, dim3(kCopyGrid), dim3(kCopyThreads), 0, s, c);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

size_t pages_workspace(int R, int num_pages) { return pg_layout(R, num_pages).bytes; }

hipError_t launch_pages_fork(const PageArgs& a, const int32_t* parent, const int32_t* child, const int32_t* len, int n,
                             void* ws, hipStream_t s) {
    const PgParams p = pg_params(a, ws);
    hipLaunchKernelGGL(pg_fork_plan, dim3(1), dim3(kPgThreads), 0, s, p, parent, child, len, n);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(pg_fork, dim3((unsigned)n), dim3(kRowThreads), 0, s, p, parent, child);
    return hipGetLastError();
}

hipError_t launch_pages_reserve(const PageArgs& a, const int32_t* cu_q, const PageBuffer* bufs, int n_bufs,
                                int32_t* step_len, void* ws, hipStream_t s) {
    const PgParams p = pg_params(a, ws);
    const unsigned chunks = (unsigned)pg_chunks(a.num_pages);
    hipLaunchKernelGGL(pg_plan, dim3(1 + chunks), dim3(kPgThreads), 0, s, p, cu_q);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(pg_assign, dim3(chunks), dim3(kPgThreads), 0, s, p, step_len);
    e = hipGetLastError();
    return e != hipSuccess ? e : copy_pages(p, bufs, n_bufs, s);
}

hipError_t launch_pages_drop(const PageArgs& a, const int32_t* step_len, const int32_t* cu_q, const int32_t* accepted,
                             const int32_t* new_len, hipStream_t s) {
    hipLaunchKernelGGL(pg_drop, dim3((unsigned)a.R), dim3(kRowThreads), 0, s, a, step_len, cu_q, accepted, new_len);
    return hipGetLastError();
}

hipError_t launch_pages_compact(const PageArgs& a, const PageBuffer* bufs, int n_bufs, int32_t* used, void* ws,
                                hipStream_t s) {
    const PgParams p = pg_params(a, ws);
    const unsigned chunks = (unsigned)pg_chunks(a.num_pages);
    hipLaunchKernelGGL(pg_count, dim3(chunks), dim3(kPgThreads), 0, s, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(pg_rank, dim3(chunks), dim3(kPgThreads), 0, s, p, used);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    // at most every second page moves
    const unsigned movers = (unsigned)(((int64_t)a.num_pages / 2 + kRowThreads - 1) / kRowThreads);
    hipLaunchKernelGGL(pg_follow, dim3((unsigned)a.R + movers), dim3(kRowThreads), 0, s, p);
    e = hipGetLastError();
    return e != hipSuccess ? e : copy_pages(p, bufs, n_bufs, s);
}

}  // namespace dspark
