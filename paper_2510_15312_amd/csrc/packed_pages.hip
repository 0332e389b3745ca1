// Requests that branch, are cut back or move to another pool: block tables, free list and share counts of a page pool on the
// device, and the copies that follow from them.  (Pages for new tokens: packed.hip.)
#include <algorithm>

#include "vf_internal.h"

namespace {

constexpr int FORK_THREADS = 256, FORK_ENTRIES = 4;   // table entries a thread
constexpr int LIST_THREADS = 1024, LIST_ENTRIES = 4;  // of the kernels that run as one workgroup

struct PagesArgs {
    int32_t n_seqs, max_pages, table_stride, pool_pages, free_entries;
};

__device__ __forceinline__ int pages_of(int tokens) { return (int)(((long long)tokens + VF_TILE - 1) / VF_TILE); }
// Tokens that a sequence holds: a negative length is none, one past the table is a full table.
__device__ __forceinline__ int held_of(int len, const PagesArgs &a) { return min(max(len, 0), a.max_pages * VF_TILE); }
__device__ __forceinline__ bool in_pool(int page, const PagesArgs &a) { return page >= 0 && page < a.pool_pages; }

// Largest i in [0, n) with v[i] <= x, for rising v with v[0] <= x.
__device__ __forceinline__ int last_not_above(const int *v, int n, int x) {
    int lo = 0;
    for (int hi = n; hi - lo > 1;) {
        const int mid = (lo + hi) >> 1;
        if (v[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Sum of v over this thread and those before it; `total` over the workgroup.  wave_sums: LDS, THREADS / 64 entries.
template <int THREADS> __device__ __forceinline__ int scan(int v, int *wave_sums, int &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int w = __shfl_up(v, d, 64);
        if (lane >= d) v += w;
    }
    if (lane == 63) wave_sums[wave] = v;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i) {
        if (i < wave) v += wave_sums[i];
        total += wave_sums[i];
    }
    __syncthreads();
    return v;
}

// ---- forks -----------------------------------------------------------------------------------------

struct ForkArgs {
    PagesArgs p;
    int32_t n_forks;
    const int32_t *src, *dst, *tokens, *len, *free_pages, *n_free;
    int32_t *table, *shares, *kv_len, *n_free_out, *copies, *n_copies;
};

// Two prefix sums over the forks (pages of their own, table entries that they share; the latter stay in LDS for the search) say where everything goes;
// every workgroup takes them for itself and then its share of the entries, so there is one launch.  The lengths go to an array of their own, as
// others still read the old ones.  Bound by the way from one read to the next (forks, lengths, last pages, entries): 4 forks of 1000
// tokens 4.0 us, 64 of 1400 7.1, 2048 of 3840 about 16 with 122,880 entries.
__global__ __launch_bounds__(FORK_THREADS) void pages_fork_kernel(ForkArgs a) {
    extern __shared__ int lds[];
    int *entries = lds, *taker = lds + a.n_forks + 1;    // entries that go before fork i's; the first fork into sequence b
    __shared__ int wave_sums[FORK_THREADS / 64];
    const PagesArgs &p = a.p;
    const int tid = threadIdx.x, nf = a.n_forks;
    const int n_free = min(max(a.n_free[0], 0), p.free_entries);
    for (int b = tid; b < p.n_seqs; b += FORK_THREADS) taker[b] = nf;
    if (tid == 0) entries[0] = 0;
    __syncthreads();
    for (int i = tid; i < nf; i += FORK_THREADS) {
        const int d = a.dst[i];
        if (d >= 0 && d < p.n_seqs) atomicMin(&taker[d], i);
    }
    __syncthreads();
    int own_before = 0, entries_before = 0;
    for (int i0 = 0; i0 < nf; i0 += FORK_THREADS) {
        const int i = i0 + tid;
        const int s = i < nf ? a.src[i] : -1, d = i < nf ? a.dst[i] : -1, want = i < nf ? a.tokens[i] : 0;
        bool ok = s >= 0 && s < p.n_seqs && d >= 0 && d < p.n_seqs;
        int t = 0;
        if (ok) {
            const int h = held_of(a.len[s], p);
            t = want < 0 || want > h ? h : want;
            ok = taker[d] == i && a.len[d] <= 0;
        }
        const bool needs = ok && t % VF_TILE && in_pool(a.table[(size_t)s * p.table_stride + t / VF_TILE], p);
        int total;
        const int upto = own_before + scan<FORK_THREADS>(needs, wave_sums, total);
        own_before += total;
        const bool granted = ok && (!needs || upto <= n_free);
        const int upto_entries = entries_before + scan<FORK_THREADS>(granted ? t / VF_TILE : 0, wave_sums, total);
        entries_before += total;
        if (i < nf) {
            entries[i + 1] = upto_entries;
            if (blockIdx.x == 0 && d >= 0 && d < p.n_seqs && taker[d] == i) {
                a.kv_len[d] = granted ? t : a.len[d];
                if (granted && t % VF_TILE) {     // the last page, of which the fork gets a copy
                    const int from = a.table[(size_t)s * p.table_stride + t / VF_TILE];
                    const int to = needs ? a.free_pages[n_free - upto] : from;
                    a.table[(size_t)d * p.table_stride + t / VF_TILE] = to;
                    if (needs) {
                        a.copies[2 * (upto - 1)] = from;
                        a.copies[2 * (upto - 1) + 1] = to;
                    }
                }
            }
        }
    }
    __syncthreads();
    if (blockIdx.x == 0) {
        for (int b = tid; b < p.n_seqs; b += FORK_THREADS)
            if (taker[b] == nf) a.kv_len[b] = a.len[b];
        if (tid == 0) {
            const int used = min(own_before, n_free);
            a.n_copies[0] = used;
            a.n_free_out[0] = n_free - used;
        }
    }
    const int step = gridDim.x * FORK_THREADS;
    for (int e = blockIdx.x * FORK_THREADS + tid; e < entries_before; e += step) {
        const int i = last_not_above(entries, nf + 1, e), t = e - entries[i];
        const int page = a.table[(size_t)a.src[i] * p.table_stride + t];
        a.table[(size_t)a.dst[i] * p.table_stride + t] = page;
        if (in_pool(page, p)) atomicAdd(&a.shares[page], 1);
    }
}

// ---- tokens that stay, pages that go back ------------------------------------------------------------

struct KeepArgs {
    PagesArgs p;
    const int32_t *len, *keep, *n_free;
    int32_t *free_pages, *table, *shares, *kv_len, *n_free_out, *copies, *n_copies;
};

__device__ __forceinline__ int now(const int32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// A barrier behind which the workgroup's atomics have been done.
__device__ __forceinline__ void done() {
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
    __syncthreads();
}

// One workgroup, whose barriers separate the steps: (1) every table entry behind what its sequence keeps drops its hold of its page
// (shares - 1); (2) a page that nobody holds any more (shares < 0) goes on the free list where the first entry that named it stands;
// (3) sequences cut inside a page that others hold drop their hold of it too and get a page of their own, but for the last of them
// where nobody else is left.  Counts are added up with atomics, whose order does not matter; who is first or last is settled by a
// minimum over the entries' numbers, kept in the (negative) count itself.  That step is left out where no page was dropped twice, and
// the third where no sequence is cut inside a page.
// What bounds it is the way from one step to the next, a trip to the L2 each, so a thread keeps the pages of its entries and of its sequences
// (of the first LIST_THREADS * LIST_ENTRIES; more are read again): 24 forks with 400 pages given back 7.5 us, 64 cut inside shared pages 11.6.
// Beyond some thousand entries the one compute unit's rate of scattered accesses bounds it, 0.45 entries a ns (60,000 pages 145 us, shared 209):
// that many end at once only when a thousand long requests do.
__global__ __launch_bounds__(LIST_THREADS) void pages_keep_kernel(KeepArgs a) {
    extern __shared__ int lds[];
    const PagesArgs &p = a.p;
    const int tid = threadIdx.x, n = p.n_seqs;
    int *start = lds, *first = lds + n + 1;     // entries that go before sequence b's; the first page that it drops
    __shared__ int wave_sums[LIST_THREADS / 64], twice, cuts;
    constexpr int FIRST = -0x7fffffff - 1;      // a count that names entry e: FIRST + e
    constexpr int EACH = VF_PACKED_MAX_SEQS / LIST_THREADS;
    if (tid == 0) start[0] = twice = cuts = 0;
    int gone = 0, n_free = min(max(a.n_free[0], 0), p.free_entries);
    int kept[EACH], cut[EACH];                  // sequence tid + i * LIST_THREADS: what it keeps; the page that it is cut inside, or -1
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        kept[i] = 0;
        cut[i] = -1;
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (i * LIST_THREADS >= n) break;
        const int b = tid + i * LIST_THREADS;
        const int h = b < n ? held_of(a.len[b], p) : 0, w = b < n ? a.keep[b] : -1, k = w < 0 || w > h ? h : w;
        if (b < n && k < h && k % VF_TILE) {
            cut[i] = a.table[(size_t)b * p.table_stride + k / VF_TILE];
            if (!in_pool(cut[i], p)) cut[i] = -1;
        }
        kept[i] = k;
        int total;
        const int upto = gone + scan<LIST_THREADS>(pages_of(h) - pages_of(k), wave_sums, total);
        gone += total;
        if (b < n) {
            start[b + 1] = upto;
            first[b] = pages_of(k);
        }
        if (cut[i] >= 0) cuts = 1;
    }
    __syncthreads();
    constexpr int CHUNK = LIST_THREADS * LIST_ENTRIES;
    int page[LIST_ENTRIES];                     // of the entries e0 + tid * LIST_ENTRIES + i
    int32_t *entry[LIST_ENTRIES];
    auto pages_from = [&](int e0) {
        const int e1 = e0 + tid * LIST_ENTRIES;
        int b = e1 < gone ? last_not_above(start, n + 1, e1) : n;
#pragma unroll
        for (int i = 0; i < LIST_ENTRIES; ++i) {
            while (b < n && e1 + i >= start[b + 1]) ++b;
            entry[i] = b < n ? a.table + (size_t)b * p.table_stride + first[b] + (e1 + i - start[b]) : nullptr;
        }
#pragma unroll
        for (int i = 0; i < LIST_ENTRIES; ++i) page[i] = entry[i] ? *entry[i] : -1;
#pragma unroll
        for (int i = 0; i < LIST_ENTRIES; ++i)
            if (!in_pool(page[i], p)) page[i] = -1;
    };
    for (int e0 = 0; e0 < gone; e0 += CHUNK) {
        pages_from(e0);
        int shared = 0;
#pragma unroll
        for (int i = 0; i < LIST_ENTRIES; ++i)
            if (page[i] >= 0) shared |= atomicSub(&a.shares[page[i]], 1);
        if (shared) twice = 1;      // a page that others hold, or that another entry has dropped
    }
    done();
    const bool settle = twice, again = gone > CHUNK;
    if (settle) {
        for (int e0 = 0; e0 < gone; e0 += CHUNK) {
            if (again) pages_from(e0);
            int s[LIST_ENTRIES];
#pragma unroll
            for (int i = 0; i < LIST_ENTRIES; ++i) s[i] = page[i] >= 0 ? now(&a.shares[page[i]]) : 0;
#pragma unroll
            for (int i = 0; i < LIST_ENTRIES; ++i)
                if (s[i] < 0) atomicMin(&a.shares[page[i]], FIRST + e0 + tid * LIST_ENTRIES + i);
        }
        done();
    }
    for (int e0 = 0; e0 < gone; e0 += CHUNK) {
        if (again) pages_from(e0);
        int s[LIST_ENTRIES], mine = 0;
#pragma unroll
        for (int i = 0; i < LIST_ENTRIES; ++i) s[i] = page[i] >= 0 ? now(&a.shares[page[i]]) : 0;
#pragma unroll
        for (int i = 0; i < LIST_ENTRIES; ++i) {
            if (entry[i]) *entry[i] = -1;
            if (s[i] >= 0 || (settle && s[i] != FIRST + e0 + tid * LIST_ENTRIES + i)) page[i] = -1;
            else ++mine;
        }
        int total, at = n_free + scan<LIST_THREADS>(mine, wave_sums, total) - mine;     // (no page is reset before all have looked)
        n_free += total;
#pragma unroll
        for (int i = 0; i < LIST_ENTRIES; ++i)
            if (page[i] >= 0) {
                a.shares[page[i]] = 0;
                if (at < p.free_entries) a.free_pages[at] = page[i];
                ++at;
            }
        if (again) done();
    }
    n_free = min(n_free, p.free_entries);
    int copied = 0;
    if (cuts) {
        done();
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (cut[i] >= 0) atomicSub(&a.shares[cut[i]], 1);
        done();
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (cut[i] >= 0 && now(&a.shares[cut[i]]) < 0) atomicMin(&a.shares[cut[i]], FIRST + (n - 1 - (tid + i * LIST_THREADS)));
        done();
        bool stays[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) stays[i] = cut[i] >= 0 && now(&a.shares[cut[i]]) == FIRST + (n - 1 - (tid + i * LIST_THREADS));
        __syncthreads();
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (i * LIST_THREADS >= n) break;
            const bool copies = cut[i] >= 0 && !stays[i];
            if (stays[i]) a.shares[cut[i]] = 0;
            int total;
            const int upto = copied + scan<LIST_THREADS>(copies, wave_sums, total);
            copied += total;
            if (copies) {
                const bool room = upto <= n_free;
                const int to = room ? a.free_pages[n_free - upto] : -1;
                a.table[(size_t)(tid + i * LIST_THREADS) * p.table_stride + kept[i] / VF_TILE] = to;
                if (room) {
                    a.copies[2 * (upto - 1)] = cut[i];
                    a.copies[2 * (upto - 1) + 1] = to;
                } else {
                    kept[i] = kept[i] / VF_TILE * VF_TILE;
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (tid + i * LIST_THREADS < n) a.kv_len[tid + i * LIST_THREADS] = kept[i];
    if (tid == 0) {
        const int used = min(copied, n_free);
        a.n_copies[0] = used;
        a.n_free_out[0] = n_free - used;
    }
}

// ---- all held pages, to a pool of their own -----------------------------------------------------------

struct CompactArgs {
    PagesArgs p;
    int32_t room, table_out_stride;
    const int32_t *len, *table, *shares;
    int32_t *table_out, *shares_out, *free_out, *n_free_out, *moved, *copies, *n_copies;
};

// One workgroup: a bit per page in LDS says which are held, and the held pages below a page are its new number.  6 sequences of a pool of 48
// pages 4.2 us, 32 of one of 889 7.6: launch, lengths, table, then the bits; next to the copies that follow (32 sequences of 1.5B: 443 us) it is little.
// Its time goes with the table's entries, all of which it visits twice, and not with the pages held: 4096 sequences x 60 entries 250 us with two
// pages each and 531 full, 256 x 2048 305 with four pages each and 716 half full.
__global__ __launch_bounds__(LIST_THREADS) void pages_compact_kernel(CompactArgs a) {
    extern __shared__ int lds[];
    const PagesArgs &p = a.p;
    const int tid = threadIdx.x, words = (p.pool_pages + 31) / 32, per = (words + LIST_THREADS - 1) / LIST_THREADS;
    unsigned *held = reinterpret_cast<unsigned *>(lds);
    __shared__ int wave_sums[LIST_THREADS / 64], before[LIST_THREADS];   // held pages before the words of a thread
    for (int w = tid; w < words; w += LIST_THREADS) held[w] = 0;
    __syncthreads();
    const int entries = p.n_seqs * p.max_pages;
    auto there = [&](int e) {    // the page of a table entry, -1 where it is none
        const int b = e / p.max_pages, t = e - b * p.max_pages;
        if (t >= pages_of(held_of(a.len[b], p))) return -1;
        const int page = a.table[(size_t)b * p.table_stride + t];
        return in_pool(page, p) ? page : -1;
    };
#pragma unroll 4
    for (int e = tid; e < entries; e += LIST_THREADS)
        if (const int page = there(e); page >= 0) atomicOr(&held[page >> 5], 1u << (page & 31));
    __syncthreads();
    int mine = 0, live;
    for (int w = tid * per; w < min(words, (tid + 1) * per); ++w) mine += __popc(held[w]);
    before[tid] = scan<LIST_THREADS>(mine, wave_sums, live) - mine;
    __syncthreads();
    auto number = [&](int page) {    // the page's new number, -1 where nobody holds it or there is no room
        const int w = page >> 5;
        const unsigned bits = held[w];
        if (!(bits >> (page & 31) & 1)) return -1;
        int rank = before[w / per] + __popc(bits & ((1u << (page & 31)) - 1));
        for (int i = w / per * per; i < w; ++i) rank += __popc(held[i]);
        return rank < a.room ? rank : -1;
    };
    for (int page = tid; page < p.pool_pages; page += LIST_THREADS) {
        const int to = number(page);
        a.moved[page] = to;
        if (to >= 0) {
            a.copies[2 * to] = page;
            a.copies[2 * to + 1] = to;
            a.shares_out[to] = a.shares[page];
        }
    }
    for (int i = live + tid; i < a.room; i += LIST_THREADS) {
        a.shares_out[i] = 0;
        a.free_out[i - live] = i;
    }
    if (tid == 0) {
        a.n_copies[0] = min(live, a.room);
        a.n_free_out[0] = max(0, a.room - live);
    }
#pragma unroll 4
    for (int e = tid; e < entries; e += LIST_THREADS) {
        const int page = there(e), b = e / p.max_pages;
        a.table_out[(size_t)b * a.table_out_stride + (e - b * p.max_pages)] = page >= 0 ? number(page) : -1;
    }
}

// ---- copies of pages -----------------------------------------------------------------------------------

// Bound by memory: 593 pages of 28 layers of 64 KB, 1.09 GB, 443 us = 4.92 TB/s read and written (a large copy of the library: 4.74).  Workgroups take pieces of
// 16 KB in turn, eight to a compute unit (pieces of 8 and 32 KB, 1024 and 4096 workgroups: within 1 %).  What is written goes past the caches: the
// next to read it is a layer's attention, with the weights of the layers before it in between, and the pages that several copies read
// stay there instead (64 forks of 3B 312 -> 289 us; with loads past the caches as well 340).
constexpr int COPY_PIECE = 16384;   // bytes a workgroup moves at a time: 64 a thread

typedef unsigned uint4v __attribute__((ext_vector_type(4)));

__global__ __launch_bounds__(256) void pages_copy_kernel(vf_copy_args a, const char *src, char *dst, const int32_t *__restrict__ copies,
                                                         const int32_t *__restrict__ n_copies) {
    const int pieces = (a.page_bytes + COPY_PIECE - 1) / COPY_PIECE;
    const long long n = min(max(n_copies[0], 0), a.max_copies), work = n * a.n_layers * pieces;
    for (long long w = blockIdx.x; w < work; w += gridDim.x) {
        const int i = (int)(w / ((long long)a.n_layers * pieces)), rest = (int)(w - (long long)i * a.n_layers * pieces);
        const int layer = rest / pieces, at = (rest - layer * pieces) * COPY_PIECE + threadIdx.x * 16;
        const int from = copies[2 * i], to = copies[2 * i + 1];
        if (from < 0 || from >= a.src_pages || to < 0 || to >= a.dst_pages) continue;
        const char *s = src + layer * a.src_layer_stride + (long long)from * a.page_bytes + at;
        char *d = dst + layer * a.dst_layer_stride + (long long)to * a.page_bytes + at;
        uint4v x[4];
        if (at + 3 * 4096 < a.page_bytes) {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = *reinterpret_cast<const uint4v *>(s + j * 4096);
#pragma unroll
            for (int j = 0; j < 4; ++j) __builtin_nontemporal_store(x[j], reinterpret_cast<uint4v *>(d + j * 4096));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (at + j * 4096 < a.page_bytes) *reinterpret_cast<uint4v *>(d + j * 4096) = *reinterpret_cast<const uint4v *>(s + j * 4096);
        }
    }
}

// What fork, keep and compact refuse alike.
int check(const char *name, const vf_pages_args *args) {
    if (!args) return vf_fail(VF_ERR_ARG, "%s: NULL argument", name);
    const vf_pages_args &a = *args;
    if (a.n_seqs < 1 || a.n_seqs > VF_PACKED_MAX_SEQS) return vf_fail(VF_ERR_ARG, "%s: n_seqs %d (1 to %d)", name, a.n_seqs, VF_PACKED_MAX_SEQS);
    if (a.max_pages < 1 || a.max_pages > 0x7fffffff / VF_TILE || a.table_stride < a.max_pages)
        return vf_fail(VF_ERR_ARG, "%s: max_pages %d, table_stride %d", name, a.max_pages, a.table_stride);
    if ((long long)a.n_seqs * a.max_pages > 1 << 30) return vf_fail(VF_ERR_UNSUPPORTED, "%s: table of %d x %d entries", name, a.n_seqs, a.max_pages);
    if (a.pool_pages < 1 || a.free_entries < 0 || a.free_entries > 0x7fffffff / VF_TILE)
        return vf_fail(VF_ERR_ARG, "%s: pool_pages %d, free_entries %d", name, a.pool_pages, a.free_entries);
    if (a.pool_pages > VF_PAGES_MAX_POOL) return vf_fail(VF_ERR_UNSUPPORTED, "%s: %d pages (at most %d)", name, a.pool_pages, VF_PAGES_MAX_POOL);
    return VF_OK;
}
PagesArgs pages_args(const vf_pages_args &a) { return {a.n_seqs, a.max_pages, a.table_stride, a.pool_pages, a.free_entries}; }

}  // namespace

extern "C" {

int vf_pages_fork(const vf_pages_args *args, int n_forks, const int32_t *src_dev, const int32_t *dst_dev, const int32_t *tokens_dev,
                  const int32_t *len_dev, const int32_t *free_pages_dev, const int32_t *n_free_dev, int32_t *block_table_dev,
                  int32_t *shares_dev, int32_t *kv_len_dev, int32_t *n_free_out_dev, int32_t *copies_dev, int32_t *n_copies_dev,
                  void *stream) {
    if (const int rc = check("vf_pages_fork", args)) return rc;
    if (n_forks < 0 || n_forks > VF_PACKED_MAX_SEQS) return vf_fail(VF_ERR_ARG, "vf_pages_fork: n_forks %d (0 to %d)", n_forks, VF_PACKED_MAX_SEQS);
    if (((!src_dev || !dst_dev || !tokens_dev || !copies_dev) && n_forks) || !len_dev || (!free_pages_dev && args->free_entries) || !n_free_dev ||
        !block_table_dev || !shares_dev || !kv_len_dev || !n_free_out_dev || !n_copies_dev)
        return vf_fail(VF_ERR_ARG, "vf_pages_fork: NULL argument");
    if (kv_len_dev == len_dev || n_free_out_dev == n_free_dev) return vf_fail(VF_ERR_ARG, "vf_pages_fork: an output is an input");
    const ForkArgs a = {pages_args(*args), n_forks, src_dev, dst_dev, tokens_dev, len_dev, free_pages_dev, n_free_dev, block_table_dev, shares_dev,
                        kv_len_dev, n_free_out_dev, copies_dev, n_copies_dev};
    const long long each = FORK_THREADS * FORK_ENTRIES;
    const int blocks = (int)std::max(1ll, std::min(256ll, ((long long)n_forks * args->max_pages + each - 1) / each));
    hipLaunchKernelGGL(pages_fork_kernel, dim3(blocks), dim3(FORK_THREADS), (size_t)(n_forks + 1 + args->n_seqs) * sizeof(int),
                       (hipStream_t)stream, a);
    VF_LAUNCH_CHECK("pages_fork");
    return VF_OK;
}

int vf_pages_keep(const vf_pages_args *args, const int32_t *len_dev, const int32_t *keep_dev, int32_t *free_pages_dev,
                  const int32_t *n_free_dev, int32_t *block_table_dev, int32_t *shares_dev, int32_t *kv_len_dev,
                  int32_t *n_free_out_dev, int32_t *copies_dev, int32_t *n_copies_dev, void *stream) {
    if (const int rc = check("vf_pages_keep", args)) return rc;
    if (!len_dev || !keep_dev || (!free_pages_dev && args->free_entries) || !n_free_dev || !block_table_dev || !shares_dev || !kv_len_dev ||
        !n_free_out_dev || !copies_dev || !n_copies_dev)
        return vf_fail(VF_ERR_ARG, "vf_pages_keep: NULL argument");
    if (kv_len_dev == len_dev || kv_len_dev == keep_dev || n_free_out_dev == n_free_dev)
        return vf_fail(VF_ERR_ARG, "vf_pages_keep: an output is an input");
    const KeepArgs a = {pages_args(*args), len_dev, keep_dev, n_free_dev, free_pages_dev, block_table_dev, shares_dev, kv_len_dev, n_free_out_dev,
                        copies_dev, n_copies_dev};
    hipLaunchKernelGGL(pages_keep_kernel, dim3(1), dim3(LIST_THREADS), (size_t)(2 * args->n_seqs + 1) * sizeof(int), (hipStream_t)stream, a);
    VF_LAUNCH_CHECK("pages_keep");
    return VF_OK;
}

int vf_pages_compact(const vf_pages_args *args, int room, int table_out_stride, const int32_t *len_dev, const int32_t *block_table_dev,
                     const int32_t *shares_dev, int32_t *table_out_dev, int32_t *shares_out_dev, int32_t *free_out_dev,
                     int32_t *n_free_out_dev, int32_t *moved_dev, int32_t *copies_dev, int32_t *n_copies_dev, void *stream) {
    if (const int rc = check("vf_pages_compact", args)) return rc;
    if (room < 1 || table_out_stride < args->max_pages) return vf_fail(VF_ERR_ARG, "vf_pages_compact: room %d, table_out_stride %d", room, table_out_stride);
    if (room > VF_PAGES_MAX_POOL) return vf_fail(VF_ERR_UNSUPPORTED, "vf_pages_compact: room for %d pages (at most %d)", room, VF_PAGES_MAX_POOL);
    if (!len_dev || !block_table_dev || !shares_dev || !table_out_dev || !shares_out_dev || !free_out_dev || !n_free_out_dev || !moved_dev ||
        !copies_dev || !n_copies_dev)
        return vf_fail(VF_ERR_ARG, "vf_pages_compact: NULL argument");
    if (shares_out_dev == shares_dev || moved_dev == shares_dev) return vf_fail(VF_ERR_ARG, "vf_pages_compact: an output is an input");
    if (table_out_dev == block_table_dev && table_out_stride != args->table_stride)
        return vf_fail(VF_ERR_ARG, "vf_pages_compact: the table in place with another stride");
    const CompactArgs a = {pages_args(*args), room, table_out_stride, len_dev, block_table_dev, shares_dev, table_out_dev, shares_out_dev, free_out_dev,
                           n_free_out_dev, moved_dev, copies_dev, n_copies_dev};
    hipLaunchKernelGGL(pages_compact_kernel, dim3(1), dim3(LIST_THREADS), (size_t)(args->pool_pages + 31) / 32 * sizeof(int), (hipStream_t)stream, a);
    VF_LAUNCH_CHECK("pages_compact");
    return VF_OK;
}

int vf_pages_copy(const vf_copy_args *args, const void *src_dev, void *dst_dev, const int32_t *copies_dev, const int32_t *n_copies_dev,
                  void *stream) {
    if (!args) return vf_fail(VF_ERR_ARG, "vf_pages_copy: NULL argument");
    const vf_copy_args &a = *args;
    if (a.n_layers < 1 || a.page_bytes < 16 || a.page_bytes > 1 << 30 || a.src_pages < 1 || a.dst_pages < 1 || a.max_copies < 0 ||
        a.max_copies > 1 << 30)
        return vf_fail(VF_ERR_ARG, "vf_pages_copy: %d layers, %d bytes a page, %d and %d pages, %d copies", a.n_layers, a.page_bytes, a.src_pages,
                       a.dst_pages, a.max_copies);
    if (a.n_layers > 1 && (a.src_layer_stride < (int64_t)a.src_pages * a.page_bytes || a.dst_layer_stride < (int64_t)a.dst_pages * a.page_bytes))
        return vf_fail(VF_ERR_ARG, "vf_pages_copy: layers overlap (strides %lld, %lld)", (long long)a.src_layer_stride, (long long)a.dst_layer_stride);
    if (a.max_copies == 0) return VF_OK;
    if (!src_dev || !dst_dev || !copies_dev || !n_copies_dev) return vf_fail(VF_ERR_ARG, "vf_pages_copy: NULL argument");
    if ((a.page_bytes | a.src_layer_stride | a.dst_layer_stride | (int64_t)(uintptr_t)src_dev | (int64_t)(uintptr_t)dst_dev) & 15)
        return vf_fail(VF_ERR_UNSUPPORTED, "vf_pages_copy: addresses, pages and layers are multiples of 16 bytes");
    const long long pieces = (a.page_bytes + COPY_PIECE - 1) / COPY_PIECE;
    if ((long long)a.n_layers * pieces > 0x7fffffff) return vf_fail(VF_ERR_UNSUPPORTED, "vf_pages_copy: %d layers of %d bytes a page", a.n_layers, a.page_bytes);
    const int blocks = (int)std::min(2048ll, a.max_copies * (a.n_layers * pieces > 2048 ? 2048 : a.n_layers * pieces));
    hipLaunchKernelGGL(pages_copy_kernel, dim3(blocks), dim3(256), 0, (hipStream_t)stream, a, (const char *)src_dev, (char *)dst_dev, copies_dev, n_copies_dev);
    VF_LAUNCH_CHECK("pages_copy");
    return VF_OK;
}

}  // extern "C"
