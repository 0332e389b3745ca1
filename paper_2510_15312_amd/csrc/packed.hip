// A packed batch over the page pool: pages and slots for the tokens of a step, rotary embedding with the write to
// the cache.  (Attention: packed_attention.hip.)
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "lds_stream.h"
#include "vf_internal.h"

namespace {

// ---- pages -----------------------------------------------------------------------------------------

constexpr int ASSIGN_THREADS = 256, ASSIGN_ROWS = 4;   // rows a thread

struct AssignArgs {
    int32_t n_seqs, max_pages, table_stride, total_rows, free_entries;
    const int32_t *len, *add, *free_pages, *n_free;
    int32_t *table, *row_off, *pos, *slot, *kv_len, *n_free_out;
};

__device__ __forceinline__ int pages_of(long long tokens) { return (int)((tokens + VF_TILE - 1) / VF_TILE); }

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

// need_b pages of sequence b come off the free list behind those of the sequences before it: two prefix sums over the
// sequences (rows, pages) say where everything goes.  Every workgroup takes them for itself (at most 32 KB, from the caches)
// and then its share of the rows and of the fresh table entries, so there is one launch and nobody waits for anybody.
// Bound by the launch and the way from one read to the next (lengths, sums, free list, table): 16 single tokens 5.2 us, 200 prompts of
// 154,625 tokens 6.3 us, where a kernel that does next to nothing takes 1.6; the host needs 3.3 for a call, from Python 7.2.
__global__ __launch_bounds__(ASSIGN_THREADS) void pages_assign_kernel(AssignArgs a) {
    extern __shared__ int lds[];
    int *off = lds, *before = lds + a.n_seqs + 1;           // rows, pages of the sequences before; pages: n_seqs + 1 entries
    __shared__ long long wave_sum[2][ASSIGN_THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.n_seqs;
    const int n_free = min(max(a.n_free[0], 0), a.free_entries);
    long long rows = 0, pages = 0;                          // sums so far
    for (int b0 = 0; b0 < n; b0 += ASSIGN_THREADS) {
        const int b = b0 + tid;
        const int h = b < n ? a.len[b] : 0, w = b < n ? a.add[b] : 0;
        const long long end = (long long)h + w;
        const bool fits = h >= 0 && w >= 0 && end <= (long long)a.max_pages * VF_TILE;
        const int need = fits ? pages_of(end) - pages_of(h) : 0;
        long long r = max(w, 0), p = need;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const long long r2 = __shfl_up(r, d, 64), p2 = __shfl_up(p, d, 64);
            if (lane >= d) { r += r2; p += p2; }
        }
        if (lane == 63) { wave_sum[0][wave] = r; wave_sum[1][wave] = p; }
        __syncthreads();
        long long all_r = 0, all_p = 0;
        for (int i = 0; i < ASSIGN_THREADS / 64; ++i) {
            if (i < wave) { r += wave_sum[0][i]; p += wave_sum[1][i]; }
            all_r += wave_sum[0][i];
            all_p += wave_sum[1][i];
        }
        r += rows;
        p += pages;
        rows += all_r;
        pages += all_p;
        __syncthreads();
        if (b < n) {
            const bool granted = fits && (need == 0 || p <= n_free);
            off[b + 1] = (int)min(r, (long long)a.total_rows);
            // pages of the granted sequences: the sums stop rising at the first that is refused for want of pages, and
            // from then on only sequences that need none are granted
            before[b + 1] = (int)min(p, (long long)0x7fffffff);
            if (blockIdx.x == 0) {
                a.row_off[b + 1] = (int)min(r, (long long)a.total_rows);
                a.kv_len[b] = granted ? (int)end : 0;
            }
        }
    }
    if (tid == 0) { off[0] = 0; before[0] = 0; }
    __syncthreads();
    // pages taken: the largest sum that the free list covers
    const int used = before[last_not_above(before, n + 1, n_free)];
    if (blockIdx.x == 0 && tid == 0) {
        a.row_off[0] = 0;
        a.n_free_out[0] = n_free - used;
    }
    const int step = gridDim.x * ASSIGN_THREADS, first = blockIdx.x * ASSIGN_THREADS + tid;
    for (int e = first; e < used; e += step) {
        const int b = last_not_above(before, n + 1, e);     // the last sequence that starts at or before e: it has pages
        a.table[(size_t)b * a.table_stride + pages_of(a.len[b]) + (e - before[b])] = a.free_pages[n_free - 1 - e];
    }
    for (int r0 = first * ASSIGN_ROWS; r0 < a.total_rows; r0 += step * ASSIGN_ROWS) {
        int b = last_not_above(off, n + 1, r0);
        int h = 0, own = 0, next = 0;
        bool granted = false, known = false;
#pragma unroll
        for (int i = 0; i < ASSIGN_ROWS; ++i) {
            const int r = r0 + i;
            if (r >= a.total_rows) break;
            while (b < n && r >= off[b + 1]) { ++b; known = false; }
            int pos = -1, slot = -1;
            if (b < n) {
                if (!known) {
                    h = a.len[b];
                    const int w = a.add[b];
                    granted = h >= 0 && w >= 0 && (long long)h + w <= (long long)a.max_pages * VF_TILE &&
                              (before[b + 1] == before[b] || before[b + 1] <= n_free);
                    own = pages_of(max(h, 0));
                    next = n_free - 1 - before[b];
                    known = true;
                }
                if (granted) {
                    pos = h + (r - off[b]);
                    const int t = pos / VF_TILE;
                    const int page = t < own ? a.table[(size_t)b * a.table_stride + t] : a.free_pages[next - (t - own)];
                    slot = page < 0 || page > 0x7fffffff / VF_TILE - 1 ? -1 : page * VF_TILE + pos % VF_TILE;
                }
            }
            a.pos[r] = pos;
            a.slot[r] = slot;
        }
    }
}

// ---- rotary embedding and the write to the cache -------------------------------------------------

__global__ void rotary_table_kernel(float2 *__restrict__ table, vf_rotary_plan p, int half) {
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= p.max_positions * half) return;
    const int pos = i / half, j = i % half;
    const double turn = 6.283185307179586476925;
    double theta = p.theta;
    if (p.scaling == VF_ROTARY_BASE) theta *= pow(p.factor, (double)p.rotary_dim / (p.rotary_dim - 2));
    double f = pow(theta, -2.0 * j / p.rotary_dim);
    if (p.scaling == VF_ROTARY_POSITIONS) f /= p.factor;
    if (p.scaling == VF_ROTARY_RAMP) {
        const double g = fmin(fmax((p.trained * f / turn - p.low) / (p.high - p.low), 0.0), 1.0);
        f *= g + (1.0 - g) / p.factor;
    }
    double s, c;
    sincos(pos * f, &s, &c);
    table[i] = make_float2((float)(c * p.magnitude), (float)(s * p.magnitude));
}

template <typename T> __device__ __forceinline__ Eight<T> eight(const T *p) { return *reinterpret_cast<const Eight<T> *>(p); }
template <typename T> __device__ __forceinline__ void put_eight(T *p, const Eight<T> &x) { *reinterpret_cast<Eight<T> *>(p) = x; }

// Sixteen elements of a head are a unit: eight pairs, which lie in two pieces of eight elements rotary_dim / 2 apart
// (half) or next to one another (interleaved, and behind rotary_dim, where nothing turns).
struct Unit { int lo, hi; bool turns; };
__device__ __forceinline__ Unit unit_of(int u, int rotary_dim, bool half) {
    const bool turns = u * 16 < rotary_dim;
    if (half && turns) return {u * 8, rotary_dim / 2 + u * 8, true};
    return {u * 16, u * 16 + 8, turns};
}
// x: eight elements of the unit's lower piece, eight of its upper one
__device__ __forceinline__ void turn_unit(float *x, const float2 *angle, bool half) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 a = angle[i];
        const int p = half ? i : 2 * i, q = half ? 8 + i : 2 * i + 1;
        const float lo = x[p] * a.x - x[q] * a.y, hi = x[q] * a.x + x[p] * a.y;
        x[p] = lo;
        x[q] = hi;
    }
}

// What bounds it is memory, and how the cache is written.  A page keeps four consecutive tokens' eight-element pieces of K next
// to one another and those of tokens 8 further behind them, and eight consecutive tokens of one feature of V.  So there are
// three kinds of workgroups: 16 rows of some heads of q, lanes along the row; the same of k, lanes along the tokens; and 64 rows
// of one head of v, which go through LDS to be written as pieces of eight tokens; v, with the longest way, comes first.  Workgroups of
// k and v whose rows are neighbours run on one die, whose L2 joins what they write to one line.  A thread of q and k keeps its row's angles
// over BATCH heads and asks for all their pieces before it turns the first.
// 8192 rows of 24 + 2 x 8 heads of 128: 39.3 us = 4.4 TB/s where a large copy reaches 4.8; 16 rows at 1.5B 3.1 us, the launch,
// the position (for k the slot too), then angles and elements, which are asked for together.
constexpr int ROTARY_ROWS = 16, ROTARY_V_ROWS = 64;

struct RotaryGrid { int32_t heads, v, k, v_rows, v_single; };   // heads a workgroup of q or k; workgroups of v, of k; rows a workgroup of v; each by itself

// Norms of q and k before they turn: a sum of squares over a head, which lies in neighbouring lanes of a wavefront, and a gain for each element.
// That takes registers, so BATCH is 2 with them (8192 rows of 24 + 2 x 8 heads of 128: 41.7 us with four heads at a time, 38.8 with two, 47.4 with
// eight) and 4 without.  Gains for every head are read when the head's sum is there, one more trip for each (float32, 1100 rows 4.8 us in a graph).
struct HeadNorms { static constexpr int BATCH = 2; vf_head_norm n; };
struct NoNorms { static constexpr int BATCH = 4; };

template <typename T, int HD, bool HALF, typename NORM>
__device__ __forceinline__ void rotate_rows(const vf_rotary_args &a, const NORM &norm, const T *src, int64_t src_stride, const float2 *table,
                                            const int32_t *pos, const int32_t *slot, T *out, bool is_k, int row, int ui, int h, int h1) {
    constexpr int SIDE = 256 / (ROTARY_ROWS * (HD / 16)), BATCH = NORM::BATCH;   // heads side by side, heads a thread at a time
    constexpr bool NORMED = std::is_same<NORM, HeadNorms>::value;
    if (row >= a.total_rows) return;
    const Unit u = unit_of(ui, a.rotary_dim, HALF);
    const int p = pos[row], s = is_k ? slot[row] : 0;
    const bool at = p >= 0 && p < a.max_positions;
    if (is_k && (!at || s < 0 || s >= a.pool_pages * VF_TILE)) return;
    float2 angle[8];
    if (u.turns) {
        const float4 *from = reinterpret_cast<const float4 *>(table + (size_t)(at ? p : 0) * (a.rotary_dim / 2) + ui * 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 x = from[i];
            angle[2 * i] = make_float2(x.x, x.y);
            angle[2 * i + 1] = make_float2(x.z, x.w);
        }
    }
    const float *gains = nullptr;
    int gain_stride = 0;
    Eight<float> gain_lo, gain_hi;
    if constexpr (NORMED) {
        gains = is_k ? norm.n.k_gain_dev : norm.n.q_gain_dev;
        gain_stride = is_k ? norm.n.k_gain_stride : norm.n.q_gain_stride;
        if (gains) {
            gain_lo = eight(gains + u.lo);
            gain_hi = eight(gains + u.hi);
        }
    }
    src += row * src_stride;
    const int per_head = is_k ? VF_TILE * HD : HD;
    const size_t to_lo = is_k ? kv_k_index(0, 0, s / VF_TILE, a.n_kv_heads, 0, s % VF_TILE, u.lo, HD) : (size_t)(row * a.q_out_stride) + u.lo;
    const size_t to_hi = is_k ? kv_k_index(0, 0, s / VF_TILE, a.n_kv_heads, 0, s % VF_TILE, u.hi, HD) : (size_t)(row * a.q_out_stride) + u.hi;
    for (; h < h1; h += BATCH * SIDE) {
        Eight<T> lo[BATCH], hi[BATCH];
        auto load = [&](int i) {
            const T *x = src + (h + i * SIDE) * HD;
            lo[i] = eight(x + u.lo);
            hi[i] = eight(x + u.hi);
        };
        if (h + (BATCH - 1) * SIDE < h1) {   // (loads with conditions of their own would be waited for all together)
#pragma unroll
            for (int i = 0; i < BATCH; ++i) load(i);
        } else {
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (h + i * SIDE < h1) load(i);
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int head = h + i * SIDE;
            if (head >= h1) break;
            if (NORMED || u.turns) {
                float x[16];
#pragma unroll
                for (int j = 0; j < 8; ++j) { x[j] = to_f32(lo[i].v[j]); x[8 + j] = to_f32(hi[i].v[j]); }
                if constexpr (NORMED) {
                    float sum = 0.f;
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum += x[j] * x[j];
                    // the head's other units are the neighbouring lanes (q), or eight or sixteen lanes apart (k)
#pragma unroll
                    for (int d = 1; d < HD / 16; d <<= 1) sum += __shfl_xor(sum, is_k ? d * (64 / (HD / 16)) : d, 64);
                    const float scale = 1.0f / sqrtf(sum * (1.0f / HD) + norm.n.eps);
                    if (gain_stride) {
                        gain_lo = eight(gains + (size_t)head * gain_stride + u.lo);
                        gain_hi = eight(gains + (size_t)head * gain_stride + u.hi);
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        x[j] *= scale;
                        x[8 + j] *= scale;
                        if (gains) {
                            x[j] *= gain_lo.v[j];
                            x[8 + j] *= gain_hi.v[j];
                        }
                    }
                }
                if (u.turns) turn_unit(x, angle, HALF);
#pragma unroll
                for (int j = 0; j < 8; ++j) { lo[i].v[j] = from_f32<T>(x[j]); hi[i].v[j] = from_f32<T>(x[8 + j]); }
            }
            if (!at) lo[i] = hi[i] = Eight<T>{};
            put_eight(out + to_lo + (size_t)head * per_head, lo[i]);
            put_eight(out + to_hi + (size_t)head * per_head, hi[i]);
        }
    }
}

template <typename T, int HD, bool HALF, typename NORM>
__global__ __launch_bounds__(256) void rotary_append_kernel(vf_rotary_args a, NORM norm, RotaryGrid g, const T *q, const T *__restrict__ k,
                                                            const T *__restrict__ v, const float2 *__restrict__ table,
                                                            const int32_t *__restrict__ pos, const int32_t *__restrict__ slot,
                                                            T *q_out, T *__restrict__ kv) {
    constexpr int UNITS = HD / 16, SIDE = 256 / (ROTARY_ROWS * UNITS);
    const int hq = a.n_q_heads, hkv = a.n_kv_heads, tid = threadIdx.x;
    int w = blockIdx.x;
    if (w >= g.k + g.v) {
        w -= g.k + g.v;
        const int per = (hq + g.heads - 1) / g.heads, h0 = w % per * g.heads;
        rotate_rows<T, HD, HALF>(a, norm, q, a.q_stride, table, pos, slot, q_out, false, w / per * ROTARY_ROWS + tid / (UNITS * SIDE), tid % UNITS,
                                 h0 + tid / UNITS % SIDE, min(h0 + g.heads, hq));
        return;
    }
    if (w >= g.v) {
        w = die_order(w - g.v, g.k);
        const int per = (hkv + g.heads - 1) / g.heads, h0 = w % per * g.heads;
        // a head's units in one wavefront where they are summed over
        const int across = std::is_same<NORM, HeadNorms>::value ? 64 / UNITS : ROTARY_ROWS;
        const int row = tid % across + tid / (across * UNITS) % (ROTARY_ROWS / across) * across;
        rotate_rows<T, HD, HALF>(a, norm, k, a.k_stride, table, pos, slot, kv, true, w / per * ROTARY_ROWS + row, tid / across % UNITS,
                                 h0 + tid / (ROTARY_ROWS * UNITS), min(h0 + g.heads, hkv));
        return;
    }
    w = die_order(w, g.v);
    const int head = w % hkv, r0 = w / hkv * g.v_rows, n_slots = a.pool_pages * VF_TILE;
    v += head * HD;
    kv += (size_t)(hkv + head) * VF_TILE * HD;
    const size_t page_size = (size_t)2 * hkv * VF_TILE * HD;
    auto slot_of = [&](int row) {   // -1: not stored
        if (row < 0 || row >= a.total_rows) return -1;
        const int p = pos[row], s = slot[row];
        return p >= 0 && p < a.max_positions && s >= 0 && s < n_slots ? s : -1;
    };
    auto place = [&](int s, int d) { return (size_t)(s / VF_TILE) * page_size + kv_v_index(0, 0, 0, 0, 0, s % VF_TILE, d, HD); };
    if (g.v_single) {   // few rows
        const int row = r0 + tid / (HD / 8), d0 = tid % (HD / 8) * 8;
        if (tid / (HD / 8) >= g.v_rows || row >= a.total_rows) return;
        const Eight<T> x = eight(v + row * a.v_stride + d0);
        const int s = slot_of(row);
        if (s < 0) return;
#pragma unroll
        for (int e = 0; e < 8; ++e) kv[place(s, d0) + e * 8] = x.v[e];
        return;
    }
    // Rows r0 - 7 .. r0 + v_rows + 6.  Eight rows with eight slots in a row from a multiple of eight on are a run; it belongs to
    // the workgroup that has its first row.
    constexpr int PAD = HD + 16 / (int)sizeof(T);
    __shared__ __align__(16) T rows[ROTARY_V_ROWS + 7][PAD];
    __shared__ int slots[ROTARY_V_ROWS + 14];
    __shared__ int firsts[ROTARY_V_ROWS], alone[ROTARY_V_ROWS], n_firsts, n_alone;
    if (tid == 0) n_firsts = n_alone = 0;
    if (tid < g.v_rows + 14) slots[tid] = slot_of(r0 - 7 + tid);
    constexpr int MOST = ((ROTARY_V_ROWS + 7) * (HD / 8) + 255) / 256;
    const int pieces = (g.v_rows + 7) * (HD / 8);
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
        const int j = tid + i * 256, row = min(r0 + j / (HD / 8), a.total_rows - 1);
        if (j < pieces) *reinterpret_cast<Eight<T> *>(&rows[j / (HD / 8)][j % (HD / 8) * 8]) = eight(v + row * a.v_stride + j % (HD / 8) * 8);
    }
    __syncthreads();
    if (tid < g.v_rows && slots[tid + 7] >= 0) {
        const int s = slots[tid + 7], first = tid + 7 - s % 8;
        bool run = first >= 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) run = run && slots[max(first, 0) + i] == s - s % 8 + i;
        if (!run) alone[atomicAdd(&n_alone, 1)] = tid;
        else if (s % 8 == 0) firsts[atomicAdd(&n_firsts, 1)] = tid;
    }
    __syncthreads();
    for (int j = tid; j < n_firsts * HD; j += 256) {
        const int r = firsts[j / HD], d = j % HD;
        Eight<T> x;
#pragma unroll
        for (int i = 0; i < 8; ++i) x.v[i] = rows[r + i][d];
        put_eight(kv + place(slots[r + 7], d), x);
    }
    for (int j = tid; j < n_alone * HD; j += 256) {
        const int r = alone[j / HD], d = j % HD;
        kv[place(slots[r + 7], d)] = rows[r][d];
    }
}

template <typename T, int HD, typename NORM>
int launch_rotary(const char *name, const vf_rotary_args &a, const NORM &norm, const void *q, const void *k, const void *v, const float *table, const int32_t *pos,
                  const int32_t *slot, void *q_out, void *kv, hipStream_t st) {
    const int tiles = (a.total_rows + ROTARY_ROWS - 1) / ROTARY_ROWS, side = 256 / (ROTARY_ROWS * (HD / 16));
    RotaryGrid g;
    // as many heads a workgroup as leave the chip about eight workgroups a compute unit, at most a batch for a thread
    g.heads = std::min((int)std::max(1ll, (long long)tiles * (a.n_q_heads + a.n_kv_heads) / (2048 * side)), NORM::BATCH) * side;
    // v: up to 128 K elements each row by itself (777 rows of two heads of 64: 3.0 us a call for 3.4), else tiles of 64 rows, or of
    // 32 or 16 where that leaves fewer than 100 workgroups (512 rows of eight heads of 128: 5.7, 5.1, 4.8; 2000 of two: 7.2, 6.4, 6.7)
    g.v_single = (long long)a.total_rows * a.n_kv_heads * HD <= 128 * 1024;
    g.v_rows = g.v_single ? 256 / (HD / 8) : ROTARY_V_ROWS;
    while (!g.v_single && g.v_rows > 16 && (long long)((a.total_rows + g.v_rows - 1) / g.v_rows) * a.n_kv_heads < 100) g.v_rows /= 2;
    const long long n_q = (long long)tiles * ((a.n_q_heads + g.heads - 1) / g.heads), n_k = (long long)tiles * ((a.n_kv_heads + g.heads - 1) / g.heads);
    const long long n_v = (long long)((a.total_rows + g.v_rows - 1) / g.v_rows) * a.n_kv_heads, blocks = n_q + n_k + n_v;
    if (blocks > 0xffffff)
        return vf_fail(VF_ERR_UNSUPPORTED, "%s: %d rows of %d heads in one call", name, a.total_rows, a.n_q_heads + 2 * a.n_kv_heads);
    g.v = (int32_t)n_v;
    g.k = (int32_t)n_k;
    const auto kernel = a.pairs == VF_ROTARY_HALF ? rotary_append_kernel<T, HD, true, NORM> : rotary_append_kernel<T, HD, false, NORM>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, st, a, norm, g, (const T *)q, (const T *)k, (const T *)v, (const float2 *)table,
                       pos, slot, (T *)q_out, (T *)kv);
    VF_LAUNCH_CHECK("rotary_append");
    return VF_OK;
}

// Both entry points: without norms, and with.
template <typename NORM>
int rotary_append(const char *name, const vf_rotary_args *args, const NORM &norm, const void *q_dev, const void *k_dev, const void *v_dev,
                  const float *table_dev, const int32_t *pos_dev, const int32_t *slot_dev, void *q_out_dev, void *kv_layer_dev, void *stream) {
    if (!args) return vf_fail(VF_ERR_ARG, "%s: NULL argument", name);
    const vf_rotary_args &a = *args;
    if (a.dtype != VF_F32 && a.dtype != VF_BF16) return vf_fail(VF_ERR_ARG, "%s: dtype %d", name, a.dtype);
    if (a.n_q_heads < 1 || a.n_kv_heads < 1 || a.n_q_heads > 256 || a.n_kv_heads > 256)
        return vf_fail(VF_ERR_ARG, "%s: %d query heads, %d key heads", name, a.n_q_heads, a.n_kv_heads);
    if (a.head_dim != 64 && a.head_dim != 128) return vf_fail(VF_ERR_UNSUPPORTED, "%s: head_dim %d (built for 64 and 128)", name, a.head_dim);
    if (a.rotary_dim < 16 || a.rotary_dim > a.head_dim || a.rotary_dim % 16)
        return vf_fail(VF_ERR_UNSUPPORTED, "%s: rotary_dim %d of head_dim %d (multiples of 16)", name, a.rotary_dim, a.head_dim);
    if (a.pairs != VF_ROTARY_HALF && a.pairs != VF_ROTARY_INTERLEAVED) return vf_fail(VF_ERR_ARG, "%s: pairs %d", name, a.pairs);
    if constexpr (std::is_same<NORM, HeadNorms>::value) {
        const vf_head_norm &n = norm.n;
        if (!(n.eps > 0) || !std::isfinite(n.eps)) return vf_fail(VF_ERR_ARG, "%s: eps %g", name, n.eps);
        for (const int stride : {n.q_gain_stride, n.k_gain_stride})
            if (stride < 0 || (stride > 0 && stride < a.head_dim) || stride > 1 << 20)
                return vf_fail(VF_ERR_ARG, "%s: gains of the heads %d elements apart", name, stride);
        if ((n.q_gain_stride | n.k_gain_stride) & 3 || ((uintptr_t)n.q_gain_dev | (uintptr_t)n.k_gain_dev) & 15)
            return vf_fail(VF_ERR_UNSUPPORTED, "%s: addresses and strides of gains are multiples of 16 bytes", name);
    }
    if (a.total_rows < 0 || a.total_rows > VF_PACKED_MAX_ROWS || a.max_positions < 1 || a.pool_pages < 1 || a.pool_pages > 0x7fffffff / VF_TILE)
        return vf_fail(VF_ERR_ARG, "%s: %d rows, %d positions, %d pages", name, a.total_rows, a.max_positions, a.pool_pages);
    if (a.total_rows == 0) return VF_OK;
    if (!q_dev || !k_dev || !v_dev || !table_dev || !pos_dev || !slot_dev || !q_out_dev || !kv_layer_dev)
        return vf_fail(VF_ERR_ARG, "%s: NULL argument", name);
    const int es = a.dtype == VF_BF16 ? 2 : 4;
    const int64_t wq = (int64_t)a.n_q_heads * a.head_dim, wkv = (int64_t)a.n_kv_heads * a.head_dim;
    if (a.q_stride < wq || a.q_out_stride < wq || a.k_stride < wkv || a.v_stride < wkv)
        return vf_fail(VF_ERR_ARG, "%s: rows overlap (strides %lld, %lld, %lld, %lld)", name, (long long)a.q_stride,
                       (long long)a.k_stride, (long long)a.v_stride, (long long)a.q_out_stride);
    if (q_out_dev == q_dev && a.q_out_stride != a.q_stride) return vf_fail(VF_ERR_ARG, "%s: q in place with another stride", name);
    if (((a.q_stride | a.k_stride | a.v_stride | a.q_out_stride) * es | (int64_t)(uintptr_t)q_dev | (int64_t)(uintptr_t)k_dev |
         (int64_t)(uintptr_t)v_dev | (int64_t)(uintptr_t)q_out_dev | (int64_t)(uintptr_t)kv_layer_dev) & 15 || (uintptr_t)table_dev & 15)
        return vf_fail(VF_ERR_UNSUPPORTED, "%s: addresses and strides are multiples of 16 bytes", name);
    hipStream_t st = (hipStream_t)stream;
    const auto launch = a.dtype == VF_BF16 ? (a.head_dim == 128 ? launch_rotary<bf16_t, 128, NORM> : launch_rotary<bf16_t, 64, NORM>)
                                           : (a.head_dim == 128 ? launch_rotary<float, 128, NORM> : launch_rotary<float, 64, NORM>);
    return launch(name, a, norm, q_dev, k_dev, v_dev, table_dev, pos_dev, slot_dev, q_out_dev, kv_layer_dev, st);
}

}  // namespace

extern "C" {

int vf_pages_assign(int n_seqs, int max_pages, int table_stride, int total_rows, int free_entries, const int32_t *len_dev,
                    const int32_t *new_dev, const int32_t *free_pages_dev, const int32_t *n_free_dev, int32_t *block_table_dev,
                    int32_t *row_off_dev, int32_t *pos_dev, int32_t *slot_dev, int32_t *kv_len_dev, int32_t *n_free_out_dev,
                    void *stream) {
    if (n_seqs < 1 || n_seqs > VF_PACKED_MAX_SEQS) return vf_fail(VF_ERR_ARG, "vf_pages_assign: n_seqs %d (1 to %d)", n_seqs, VF_PACKED_MAX_SEQS);
    if (max_pages < 1 || max_pages > 0x7fffffff / VF_TILE || table_stride < max_pages || total_rows < 0 || total_rows > VF_PACKED_MAX_ROWS ||
        free_entries < 0 || free_entries > 0x7fffffff / VF_TILE)
        return vf_fail(VF_ERR_ARG, "vf_pages_assign: max_pages %d, table_stride %d, total_rows %d, free_entries %d", max_pages,
                       table_stride, total_rows, free_entries);
    if (!len_dev || !new_dev || (!free_pages_dev && free_entries) || !n_free_dev || !block_table_dev || !row_off_dev ||
        ((!pos_dev || !slot_dev) && total_rows) || !kv_len_dev || !n_free_out_dev)
        return vf_fail(VF_ERR_ARG, "vf_pages_assign: NULL argument");
    if (kv_len_dev == len_dev || kv_len_dev == new_dev || n_free_out_dev == n_free_dev)
        return vf_fail(VF_ERR_ARG, "vf_pages_assign: an output is an input");
    const AssignArgs a = {n_seqs, max_pages, table_stride, total_rows, free_entries, len_dev, new_dev, free_pages_dev, n_free_dev,
                          block_table_dev, row_off_dev, pos_dev, slot_dev, kv_len_dev, n_free_out_dev};
    const int blocks = std::max(1, std::min(256, (int)(((long long)total_rows + ASSIGN_THREADS * ASSIGN_ROWS - 1) / (ASSIGN_THREADS * ASSIGN_ROWS))));
    hipLaunchKernelGGL(pages_assign_kernel, dim3(blocks), dim3(ASSIGN_THREADS), (size_t)(n_seqs + 1) * 2 * sizeof(int),
                       (hipStream_t)stream, a);
    VF_LAUNCH_CHECK("pages_assign");
    return VF_OK;
}

int vf_rotary_table(const vf_rotary_plan *plan, float *table_dev, void *stream) {
    if (!plan || !table_dev) return vf_fail(VF_ERR_ARG, "vf_rotary_table: NULL argument");
    const vf_rotary_plan &p = *plan;
    if (p.rotary_dim < 16 || p.rotary_dim > 128 || p.rotary_dim % 16 || p.max_positions < 1 || p.max_positions > (1 << 24))
        return vf_fail(VF_ERR_ARG, "vf_rotary_table: rotary_dim %d, max_positions %d", p.rotary_dim, p.max_positions);
    if (!(p.theta > 0) || !std::isfinite(p.theta) || !std::isfinite(p.magnitude)) return vf_fail(VF_ERR_ARG, "vf_rotary_table: theta %g, magnitude %g", p.theta, p.magnitude);
    if (p.scaling < VF_ROTARY_UNSCALED || p.scaling > VF_ROTARY_RAMP) return vf_fail(VF_ERR_ARG, "vf_rotary_table: scaling %d", p.scaling);
    if (p.scaling != VF_ROTARY_UNSCALED && (!(p.factor > 0) || !std::isfinite(p.factor))) return vf_fail(VF_ERR_ARG, "vf_rotary_table: factor %g", p.factor);
    if (p.scaling == VF_ROTARY_RAMP && (!(p.trained > 0) || !std::isfinite(p.trained) || !(p.high > p.low) || !std::isfinite(p.high) || !std::isfinite(p.low)))
        return vf_fail(VF_ERR_ARG, "vf_rotary_table: ramp from %g to %g turns over %g positions", p.low, p.high, p.trained);
    const int half = p.rotary_dim / 2;
    const long long n = (long long)p.max_positions * half;
    hipLaunchKernelGGL(rotary_table_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, (hipStream_t)stream, (float2 *)table_dev, p, half);
    VF_LAUNCH_CHECK("rotary_table");
    return VF_OK;
}

int vf_rotary_append(const vf_rotary_args *args, const void *q_dev, const void *k_dev, const void *v_dev, const float *table_dev,
                     const int32_t *pos_dev, const int32_t *slot_dev, void *q_out_dev, void *kv_layer_dev, void *stream) {
    return rotary_append("vf_rotary_append", args, NoNorms{}, q_dev, k_dev, v_dev, table_dev, pos_dev, slot_dev, q_out_dev, kv_layer_dev, stream);
}

int vf_norm_rotary_append(const vf_rotary_args *args, const vf_head_norm *norm, const void *q_dev, const void *k_dev, const void *v_dev,
                          const float *table_dev, const int32_t *pos_dev, const int32_t *slot_dev, void *q_out_dev, void *kv_layer_dev,
                          void *stream) {
    if (!norm) return vf_fail(VF_ERR_ARG, "vf_norm_rotary_append: NULL argument");
    HeadNorms norms{*norm};
    if (!norm->q_gain_dev) norms.n.q_gain_stride = 0;
    if (!norm->k_gain_dev) norms.n.k_gain_stride = 0;
    return rotary_append("vf_norm_rotary_append", args, norms, q_dev, k_dev, v_dev, table_dev, pos_dev, slot_dev, q_out_dev, kv_layer_dev, stream);
}

}  // extern "C"
