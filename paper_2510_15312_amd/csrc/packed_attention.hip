// Causal attention of packed rows with grouped heads over the page pool: whole prompts, chunks behind a cached prefix,
// drafts and single tokens of many sequences in one call.
//
// An item at position p: o = sum_t w_t v_t / sum_t w_t over the keys t <= p, w_t = 2^(c s_t - m), s_t = q . k_t, c = scale log2(e).
// One pass over the pages keeps m, the sum of the weights and the sum of the products in float32; when m moves to m', both sums are
// taken times 2^(m - m').  Any m gives the same quotient, so that parts of the keys can be taken apart and joined by the same factor.
//
// The rows of a sequence and the query heads of one key head are its items, row-major: all items of a key head meet the same
// keys, so a tile of items reads them once whatever the group is, and few rows fill a tile as well as they can.
// With S = K Q^T (keys down, items across) a lane holds one item's scores, so the softmax is arithmetic inside a lane and one
// exchange between the wavefront's halves, and S is already the operand of O^T = V^T P^T.
//
// Three kernels: tiles of 128 items (many rows: bound by the instructions of products and softmax), the same with two groups of
// wavefronts on alternate pages (tiles that would leave the chip half empty), tiles of 16 items (few rows: bound by the cache's
// bytes and the launch).  make_plan chooses.
#include <algorithm>
#include <cmath>

#include "fast_common.h"
#include "lds_stream.h"
#include "vf_internal.h"

namespace {

// Division by a number the host knows: a multiplication that is at most one too high, put right.
struct Divisor {
    unsigned d, m;
    __device__ __forceinline__ int operator()(int n) const {   // n / d, n >= 0
        if (d == 1) return n;
        const unsigned q = __umulhi((unsigned)n, m);
        return (int)(q - (q * d > (unsigned)n));
    }
};
inline Divisor divisor(unsigned d) { return {d, d > 1 ? (unsigned)((1ull << 32) / d + 1) : 0}; }

struct PackedAttn {
    vf_packed_args a;
    const void *q, *kv;
    const int32_t *table, *row_off, *kv_len;
    void *out;
    int32_t group, tiles, parts, part_pages;   // tiles: items tiles of all sequences, at most
    int32_t tile_is_seq;                       // a tile is all items of a sequence
    int32_t by_height;                         // tiles with the most keys first
    Divisor by_group, by_heads, by_tiles, by_q_heads;
    float scale_log2e;
    float *records;                            // [row][head][part][REC_HEAD + head_dim], parts > 1
    int32_t *used;                             // [row]: parts with a record
};
constexpr int REC_HEAD = 4;                    // maximum, sum, -, -
constexpr int TILE_WAVES = 4, FEW_ITEMS = 16;
// A running maximum of no keys: the type's lowest, so that any score is above it, and 2^(LOWEST - m) is 0 beside any other m and 1
// beside itself.
constexpr float LOWEST = -3.40282347e38f;

typedef float floatx16 __attribute__((ext_vector_type(16)));

// A tile of BM items: its sequence's rows and keys.  rows <= 0: none.
struct Tile { int seq, item0, row0, rows, kv_len; };
__device__ __forceinline__ int2 seq_rows(const PackedAttn &p, int b) {   // first row and rows, whatever the offsets hold
    const int r0 = min(max(p.row_off[b], 0), p.a.total_rows), r1 = min(max(p.row_off[b + 1], r0), p.a.total_rows);
    return {r0, r1 - r0};
}
// Keys of a sequence, whatever the length holds: a negative one is none (the lowest would come out as the highest once rows are taken from it).
__device__ __forceinline__ int seq_keys(const PackedAttn &p, int b) { return max(p.kv_len[b], 0); }
// Over the wavefront's lanes, for values that are not negative: up to and with this lane.
template <int CTRL, int ROWS, typename F> __device__ __forceinline__ int lane_step(int x, F f) {
    return f(x, __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false));
}
template <typename F> __device__ __forceinline__ int lanes_upto(int x, F f) {
    x = lane_step<0x111, 0xf>(x, f);   // a row of 16 lanes: by 1, 2, 4, 8
    x = lane_step<0x112, 0xf>(x, f);
    x = lane_step<0x114, 0xf>(x, f);
    x = lane_step<0x118, 0xf>(x, f);
    x = lane_step<0x142, 0xa>(x, f);   // a row's last lane to the next row
    return lane_step<0x143, 0xc>(x, f);   // lane 31 to the upper half
}
struct Plus { __device__ __forceinline__ int operator()(int x, int y) const { return x + y; } };
struct Max { __device__ __forceinline__ int operator()(int x, int y) const { return max(x, y); } };
// Tiles of cached tokens.  Past 2^30 the order of heights does not matter, but that no height overflows does: a tile that the search
// does not find would lie outside its sequence.
__host__ __device__ constexpr int cached_tiles(int tokens, int group, int bm) {
    const long long tiles = (long long)(tokens > 0 ? tokens : 0) * group / bm;
    return tiles < (1 << 30) ? (int)tiles : 1 << 30;
}
static_assert(cached_tiles(0x7fffffff / VF_TILE * VF_TILE, 256, TILE_WAVES * 32) + (long long)VF_PACKED_MAX_ROWS * 256 / (TILE_WAVES * 32) <= 0x7fffffff &&
                  cached_tiles(0x7fffffff, 256, TILE_WAVES * 32) > 0 && cached_tiles(8192, 3, TILE_WAVES * 32) == 192 && cached_tiles(-5, 3, 128) == 0,
              "the longest sequence of the largest group");
// Tile number `tile` of all, 64 sequences at a time: sequence by sequence, or those with the most keys first (by_height).  A tile's
// height is its place in its sequence, counted in tiles, cached tokens among them; as high as h or higher are clamp(end - h, 0, tiles)
// of a sequence.
template <int BM> __device__ __forceinline__ Tile find_tile(const PackedAttn &p, int tile, bool by_height) {
    const int lane = threadIdx.x & 63;
    for (int b0 = 0; b0 < p.a.n_seqs; b0 += 64) {
        const int b = min(b0 + lane, p.a.n_seqs - 1);
        const int2 r = seq_rows(p, b);
        const int len = seq_keys(p, b);
        const int tiles = b0 + lane < p.a.n_seqs ? (int)(((long long)r.y * p.group + BM - 1) / BM) : 0;
        const int upto = lanes_upto(tiles, Plus{}), all = __builtin_amdgcn_readlane(upto, 63);
        if (tile >= all) {
            tile -= all;
            continue;
        }
        int at, place;
        if (by_height) {
            const int cached = cached_tiles(min(len - r.y, p.a.max_pages * VF_TILE), p.group, BM), end = cached + tiles;
            int low = 0, high = __builtin_amdgcn_readlane(lanes_upto(tiles ? end : 0, Max{}), 63), higher = 0;
            while (high - low > 1) {   // the tile's height is low or more and less than high; `higher` tiles are at high or higher
                const int middle = low + ((high - low) >> 1);
                const int count = __builtin_amdgcn_readlane(lanes_upto(max(0, min(end - middle, tiles)), Plus{}), 63);
                if (count > tile) low = middle;
                else high = middle, higher = count;
            }
            const unsigned long long here = __builtin_amdgcn_ballot_w64(cached <= low && low < end);
            const int rank = __builtin_amdgcn_mbcnt_hi((unsigned)(here >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)here, 0));
            at = __builtin_ctzll(here & __builtin_amdgcn_ballot_w64(rank == tile - higher));
            place = low - __builtin_amdgcn_readlane(cached, at);
        } else {
            at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > tile));
            place = __builtin_amdgcn_readlane(upto, at) - 1 - tile;   // a sequence's last rows see the most
        }
        return {b0 + at, place * BM, __builtin_amdgcn_readlane(r.x, at), __builtin_amdgcn_readlane(r.y, at), __builtin_amdgcn_readlane(len, at)};
    }
    return {0, 0, 0, 0, 0};
}

__device__ __forceinline__ float halves_max(float x) {
    float y = x;
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(x), "+v"(y));
    return fmaxf(x, y);
}
__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

// Operands of a 32x32 product over 16 values of k (32 lanes each take 8): bfloat16 in one matrix instruction, float32 in eight.
template <typename T> struct Frag;
template <> struct Frag<bf16_t> { bf16x8 v; };
template <> struct Frag<float> { float v[8]; };
__device__ __forceinline__ floatx16 mma(const Frag<bf16_t> &a, const Frag<bf16_t> &b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ floatx16 mma(const Frag<float> &a, const Frag<float> &b, floatx16 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[j], b.v[j], c, 0, 0, 0);
    return c;
}

// Four kilobytes apart by OFF from memory straight to LDS, free to be moved by the compiler: a statement takes `order` and hands it on.
// The destination goes through m0 (one idle cycle before the load); an instruction's own offset counts for both addresses.
template <int OFF> __device__ __forceinline__ int unit_to_lds(int order, const void *src, unsigned lane_off, unsigned lds) {
    if constexpr (OFF == 0) asm("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3" : "+s"(order) : "s"(lds), "v"(lane_off), "s"(src));
    else asm("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3 offset:%4" : "+s"(order) : "s"(lds), "v"(lane_off), "s"(src), "n"(OFF));
    return order;
}

// Tiles of 32 items a wavefront, pages of 64 keys through LDS.
//
// A page comes as direct loads of 1 KB units.  Units hold 16 bytes a lane: a K or V piece of eight elements
// in bfloat16, half of one in float32 (the halves of a fragment's pieces in two units, so that a read of 16 bytes a lane
// touches every bank once).  K rows are taken in the order that leaves a lane with eight consecutive keys per operand of
// the second product: row m of a 32-key tile is key 16 (m >> 4) + 8 (m >> 2 & 1) + 4 (m >> 3 & 1) + (m & 3).
//
// What bounds it: a page of heads of 128 is 32 matrix instructions of 32 cycles among 135 on vectors and about 100 scalar and LDS
// instructions of a wavefront, which issues one in four to five cycles; two wavefronts share a SIMD.  A prompt of 8192 tokens at 3B
// (24 heads of 128, 8 of K and V) takes 373 to 396 us
// = 1.04 to 1.1 PFLOP/s where a large matrix product reaches 1.3; the matrix units are busy 58 % of the cycles, at a clock that
// the power limit has brought to 1.7 GHz.  20000 tokens at 1.5B: 1.12 PFLOP/s; at 0.5B (heads of 64, whose products are half as
// long for the same softmax) 0.9.  Twelve prompts of 230 to 2048 tokens at 0.5B 59 us = 694 TFLOP/s: a tile has 16 pages on
// average, of which the last one or two are masked, behind a start of three dependent reads.
// Not taken, as no faster: three and four pages in flight, eight wavefronts on one page, a hand-laid order of the page's
// instructions, the sum of the weights by additions instead of two-term products.
// Heads of 64 in bfloat16 leave registers for a third wavefront on a SIMD, if a page's scores are not computed ahead of the page
// before: three hide more than the order of one (twelve prompts of 230 to 2048 tokens at 0.5B 67 -> 60 us, one of 16384
// 570 -> 521 us).  Heads of 128 fill the registers of two; four wavefronts spill in what comes after the full pages (68 us).
template <typename T, int HD, int KG> constexpr int tile_waves_per_simd = HD == 64 && KG == 1 && sizeof(T) == 2 ? 3 : 2;
template <typename T, int HD, int KG>
__global__ __launch_bounds__(TILE_WAVES * KG * 64, (tile_waves_per_simd<T, HD, KG>)) void attention_tiles_kernel(PackedAttn p) {
    constexpr int WAVES = TILE_WAVES, BM = WAVES * 32, HALVES = sizeof(T) / 2, UNITS = HD / 4 * HALVES, LPW = UNITS / WAVES;   // units of a page
    constexpr int KD = HD / 32, KS = HD / 16, DB = HD / 32;
    static_assert(UNITS % (2 * WAVES) == 0, "a wavefront loads K or V");
    extern __shared__ __align__(1024) unsigned char smem[];
    const vf_packed_args &a = p.a;
    const int lane = threadIdx.x & 63, any_wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, col = lane & 31;
    const int wave = any_wave % WAVES, kg = any_wave / WAVES, tid = threadIdx.x % (WAVES * 64);   // within the group of wavefronts kg
    const int rest = p.by_heads(blockIdx.x), kvh = blockIdx.x - rest * a.n_kv_heads, part = p.by_tiles(rest), place = rest - part * p.tiles;
    const Tile t = find_tile<BM>(p, place, p.by_height);
    if (t.rows <= 0) return;
    const int group = p.group, n_items = t.rows * group, cap = min(t.kv_len, a.max_pages * VF_TILE);
    const int first_pos = t.kv_len - t.rows;                    // position of row 0
    const int wave0 = t.item0 + wave * 32, item = min(n_items - 1, wave0 + col);
    const int item_row = p.by_group(item), item_head = item - item_row * group, row = t.row0 + item_row, head = kvh * group + item_head;
    const int last_key = min(first_pos + item_row, cap - 1);
    const int tile_last = min(first_pos + p.by_group(min(n_items - 1, t.item0 + BM - 1)), cap - 1);
    const int tile_first = min(first_pos + p.by_group(t.item0), cap - 1);
    const bool has_items = wave0 < n_items;   // a wavefront without items still brings its share of the pages
    const int wave_last = has_items ? min(first_pos + p.by_group(min(n_items - 1, wave0 + 31)), cap - 1) : -1;
    const int wave_first = min(first_pos + p.by_group(min(n_items - 1, wave0)), cap - 1);
    const int pages = tile_last < 0 ? 0 : tile_last / VF_TILE + 1;
    const int p_begin = part * p.part_pages, p_end = part == p.parts - 1 ? pages : min(pages, p_begin + p.part_pages);
    if (p.parts > 1 && part == 0 && kvh == 0 && wave0 + col < n_items && half == 0 && kg == 0 && item_head == 0)
        p.used[row] = min(p.parts, (pages + p.part_pages - 1) / p.part_pages);
    if (p_begin >= p_end && part > 0) return;

    Frag<T> qf[KS];
    {
        const T *q = (const T *)p.q + row * a.q_stride + head * HD + half * 8;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const Eight<T> x = *reinterpret_cast<const Eight<T> *>(q + s * 16);
#pragma unroll
            for (int j = 0; j < 8; ++j) qf[s].v[j] = x.v[j];
        }
    }
    const size_t page_bytes = (size_t)2 * a.n_kv_heads * VF_TILE * HD * sizeof(T);
    const char *src = (const char *)p.kv + (size_t)(wave < WAVES / 2 ? kvh : a.n_kv_heads + kvh) * (VF_TILE * HD * sizeof(T)) +
                      wave % (WAVES / 2) * (LPW * 1024);
    unsigned char *const pages_lds = smem + kg * (2 * UNITS * 1024);
    const unsigned lds0 = lds_address(pages_lds) + wave * (LPW * 1024);
    const int32_t *table = p.table + (size_t)t.seq * a.table_stride;
    // ids of 64 pages, one per lane: those from ids_at on.  The loads of K ask a step ahead of the products, so that a page asked
    // for may also lie in front of them.
    int ids_at = p_begin, ids = table[min(p_begin + lane, a.max_pages - 1)];
    auto page_id = [&](int pg) {
        if ((unsigned)(pg - ids_at) >= 64u) {
            ids_at = pg;
            ids = table[min(pg + lane, a.max_pages - 1)];
        }
        const int id = __builtin_amdgcn_readlane(ids, pg - ids_at);
        return (unsigned)id < (unsigned)a.pool_pages ? id : -1;
    };
    // Step i takes page p_begin + KG i + kg.  K of step i + 1 and V of step i travel together, one step ahead of their use: a
    // wavefront brings K or V.
    // The loads' statements are tied to the step's barrier by `order`, which each takes and hands on, and are otherwise free to
    // stand among the products (a volatile statement is a fence for every LDS read: 200 cycles in front of the first product).
    int order = 0;
    struct Source { const char *from; unsigned dst; };
    auto source = [&](int i) {
        const int step = i + (wave < WAVES / 2 ? 1 : 0);
        const int id = page_id(max(p_begin, min(p_begin + step * KG + kg, p_end - 1)));   // a page that is not needed: some page, not used
        return Source{src + (size_t)max(id, 0) * page_bytes, lds0 + (unsigned)(step & 1) * (UNITS * 1024)};
    };
    auto issue_unit = [&](const Source &x, auto f) {
        constexpr int F = f;
        const unsigned off = HALVES == 1 ? lane * 16 : lane * 32;
        if constexpr (HALVES == 1) order = unit_to_lds<F % 4 * 1024>(order, x.from + F / 4 * 4096, off, x.dst + F / 4 * 4096);
        else order = unit_to_lds<0>(order, x.from + F / 2 * 2048 + F % 2 * 16, off, x.dst + F * 1024);
    };
    auto issue = [&](int i) {
        const Source x = source(i);
        static_for<0, LPW>([&](auto f) { issue_unit(x, f); });
    };
    auto landed = [&](auto left) {   // until at most `left` of this wavefront's loads are outstanding, then the workgroup's barrier
        asm volatile("s_waitcnt vmcnt(%0)" : : "n"((int)left), "s"(order) : "memory");
        lds_sync();
        asm volatile("" : "+s"(order) : : "memory");
    };
    // a lane's pieces: K row col of a 32-key tile, V^T row col of 32 output dimensions
    const unsigned k_lane = (unsigned)((col >> 3 & 1) * KD * 64 * HALVES + half * 16 + (col >> 4) * 8 + (col >> 2 & 1) * 4 + (col & 3)) * 16;
    const unsigned v_lane = (unsigned)((col >> 4) * 64 * HALVES + half * 16 + (col & 15)) * 16;
    auto piece = [&](const unsigned char *at) {
        Frag<T> f;
        if constexpr (HALVES == 1) f.v = *reinterpret_cast<const bf16x8 *>(at);
        else
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const floatx4 x = *reinterpret_cast<const floatx4 *>(at + h * 1024);
#pragma unroll
                for (int j = 0; j < 4; ++j) f.v[h * 4 + j] = x[j];
            }
        return f;
    };
    auto k_piece = [&](const unsigned char *st, int kt, int s) { return piece(st + k_lane + (kt * 2 * KD + s / 2) * 1024 * HALVES + s % 2 * 512); };
    auto v_piece = [&](const unsigned char *st, int kt, int tt, int db) {
        return piece(st + UNITS / 2 * 1024 + v_lane + (kt * 2 * DB + db * 2) * 1024 * HALVES + tt * 512);
    };
    floatx16 acc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[db][i] = 0.f;
    float m_run = LOWEST, l_run = 0.f;   // l_run: this lane's keys
    // A weight's exponent is fma(score, by, -m_run), the scale inside.  m_run was rounded where the product of the fma is not, a
    // common factor of up to 2^(2^-24 |m_run|): nothing up to 2^24.  Beyond that the scores are scaled and rounded first, and `by` is 1.
    float by = p.scale_log2e;
    bool far = false;
    struct Scores { floatx16 t[2]; };   // 32 keys each: register i of t[kt] is key 32 kt + 16 (i >> 3) + 8 half + (i & 7) of the page
    auto scores = [&](const unsigned char *st) {
        Scores sc;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc.t[kt][i] = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) sc.t[kt] = mma(k_piece(st, kt, s), qf[s], sc.t[kt]);
        return sc;
    };
    Frag<T> w[4];
    // The weights' common factor follows the maximum with slack: they stay below 2^8, and the sums are rescaled in few pages.
    auto follow = [&](Scores &sc) {
        float mx = sc.t[0][0];
#pragma unroll
        for (int i = 1; i < 32; ++i) mx = fmaxf(mx, sc.t[i >> 4][i & 15]);
        mx = halves_max(mx) * p.scale_log2e;
        if (__builtin_amdgcn_ballot_w64(mx > m_run + 8.f)) {
            const float m_new = fmaxf(m_run, mx), keep = __builtin_amdgcn_exp2f(m_run - m_new);
            l_run *= keep;
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] *= keep;
            m_run = m_new;
            far = __builtin_amdgcn_ballot_w64(fabsf(m_new) > 0x1p24f && m_new != LOWEST);
            by = far ? 1.f : p.scale_log2e;
        }
        if (far) {
#pragma clang fp contract(off)
#pragma unroll
            for (int i = 0; i < 32; ++i) sc.t[i >> 4][i & 15] *= p.scale_log2e;
        }
    };
    // Weights are rounded to bfloat16 for the product with V, which is bfloat16 itself: results are off by 2.0e-3 of their size where
    // their own rounding is 1.6e-3.  A second bfloat16 value a weight, as the kernel for few items takes, would be half as many matrix
    // instructions again, and 16 registers where heads of 128 have 5 left.
    auto weights = [&](const Scores &sc) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const float x = __builtin_amdgcn_exp2f(fmaf(sc.t[i >> 4][i & 15], by, -m_run));
            if constexpr (HALVES == 2) l_run += x;
            w[i >> 3].v[i & 7] = from_f32<T>(x);
        }
        // the sum is that of the rounded weights, which the products take
        if constexpr (HALVES == 1)
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
                typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
                l_run = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{w[i >> 3].v[i & 7], w[i >> 3].v[(i & 7) + 1]}, bf16x2{(bf16_t)1.f, (bf16_t)1.f}, l_run, false);
            }
    };
    auto products = [&](const unsigned char *st) {   // O^T += V^T W^T
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] = mma(v_piece(st, g / 2, g % 2, db), w[g], acc[db]);
    };
    // The same where some keys are not seen by all items.  0 times a value that is not finite is not a number: where that comes
    // out, every row takes the product with its own keys.
    auto products_masked = [&](const unsigned char *st, int t0) {
        const int page_last = min(wave_last, t0 + VF_TILE - 1);
        static_for<0, DB>([&](auto db) {
            constexpr int D = db;
            floatx16 all = acc[D];
#pragma unroll
            for (int g = 0; g < 4; ++g) all = mma(v_piece(st, g / 2, g % 2, D), w[g], all);
            bool bad = false;
#pragma unroll
            for (int i = 0; i < 16; i += 2) bad |= __builtin_isunordered(all[i], all[i + 1]);
            if (!__builtin_amdgcn_ballot_w64(bad)) {
                acc[D] = all;
            } else {
                floatx16 sum = acc[D];   // of rows that see nothing here
                for (int seen = min(max(wave_first, t0), page_last); seen <= page_last; ++seen) {   // (all rows may see the page whole)
                    floatx16 c = acc[D];
                    int keys = seen - t0 - half * 8;   // held back, or the compiler keeps 32 comparisons' operands through the whole kernel
                    asm volatile("" : "+v"(keys));
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        Frag<T> x = v_piece(st, g / 2, g % 2, D);
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (g * 16 + j > keys) x.v[j] = from_f32<T>(0.f);
                        c = mma(x, w[g], c);
                    }
                    if (min(last_key, t0 + VF_TILE - 1) == seen) sum = c;
                }
                acc[D] = sum;
            }
            __builtin_amdgcn_sched_barrier(0);   // one block's values in registers at a time
        });
    };
    // Memory behind the last key may hold anything: its values count as zeros.
    auto clear_behind = [&](unsigned char *st, int keys) {   // keys: of the page that are there
        for (int u = tid; u < UNITS / 2 * 64; u += WAVES * 64) {
            const int piece = HALVES == 1 ? u : (u >> 7 << 6) + (u & 63), e0 = HALVES == 1 ? 0 : (u >> 6 & 1) * 4;
            const int there = keys - (piece / (DB * 128) * 32 + (piece >> 4 & 3) * 8) - e0;   // of this unit's 16 / sizeof(T) elements
            if (there >= 16 / (int)sizeof(T)) continue;
            T *x = reinterpret_cast<T *>(st + UNITS / 2 * 1024 + u * 16);
#pragma unroll
            for (int j = 0; j < 16 / (int)sizeof(T); ++j)
                if (j >= there) x[j] = from_f32<T>(0.f);
        }
    };
    // A step: a page's weights and products, and the scores of the next step's page, which do not wait for them.
    const int n = (p_end - p_begin + KG - 1) / KG;
    if (n > 0) {
        // pages that all items see whole, up to the first that is not in the pool
        int full = max(0, min(p_end - p_begin, (tile_first + 1) / VF_TILE - p_begin));
        for (int i0 = 0; i0 < full; i0 += 64) {
            const int id = i0 ? table[p_begin + min(i0 + lane, full - 1)] : ids;
            const unsigned long long missing = __builtin_amdgcn_ballot_w64(i0 + lane < full && (unsigned)id >= (unsigned)a.pool_pages);
            if (missing) full = min(full, i0 + __builtin_ctzll(missing));
        }
        const int n_full = full / KG;
        auto k_page = [&](int i) { return pages_lds + (i & 1) * (UNITS * 1024); };
        auto step = [&](int i) {   // behind it K of step i + 1 and V of step i have landed, and their slots' neighbours are free
            landed(std::integral_constant<int, 0>{});
            issue(i + 1);
        };
        auto tail = [&](int i) {   // behind a step past n_full
            if (cap - (p_begin + i * KG) * VF_TILE < VF_TILE * KG) {   // a page of the step is not full
                clear_behind(k_page(i), cap - (p_begin + i * KG + kg) * VF_TILE);
                lds_sync();
            }
        };
        issue(-1);
        issue(0);
        landed(std::integral_constant<int, LPW>{});
        if (!has_items) {
            for (int i = 0; i < n; ++i) {
                step(i);
                if (i >= n_full) tail(i);
            }
        } else {
            int i = 0;
            if constexpr (tile_waves_per_simd<T, HD, KG> == 3) {
                for (; i < n_full; ++i) {
                    Scores sc = scores(k_page(i));
                    step(i);
                    follow(sc);
                    weights(sc);
                    products(k_page(i));
                }
            } else if (n_full > 0) {
                Scores even = scores(k_page(0)), odd;
                follow(even);
                auto last = [&](const Scores &sc) {
                    step(i);
                    weights(sc);
                    products(k_page(i));
                    ++i;
                };
                auto next = [&](const Scores &sc, Scores &ahead) {
                    step(i);
                    ahead = scores(k_page(i + 1));
                    weights(sc);
                    products(k_page(i));
                    follow(ahead);
                    ++i;
                };
                while (i + 2 < n_full) {
                    next(even, odd);
                    next(odd, even);
                }
                if (i + 1 < n_full) {
                    next(even, odd);
                    last(odd);
                } else {
                    last(even);
                }
            }
            for (; i < n; ++i) {
                const int pg = p_begin + i * KG + kg, t0 = pg * VF_TILE;
                const bool mine = pg < p_end && t0 <= wave_last && page_id(min(pg, p_end - 1)) >= 0;
                Scores sc;
                if (mine) sc = scores(k_page(i));
                step(i);
                tail(i);
                if (!mine) continue;
                const int keys = last_key - t0 - half * 8;
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if ((j >> 3) * 16 + (j & 7) > keys) sc.t[j >> 4][j & 15] = -INFINITY;
                follow(sc);
                weights(sc);
                products_masked(k_page(i), t0);
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" : : "s"(order) : "memory");   // nothing is on its way to LDS when the workgroup ends
    }
    if constexpr (KG == 2) {   // the second group's sums join the first's
        float *const at = reinterpret_cast<float *>(smem) + wave * (DB * 16 + 2) * 64 + lane;
        lds_sync();
        if (kg == 1) {
            at[0] = m_run;
            at[64] = l_run;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) at[(2 + db * 16 + i) * 64] = acc[db][i];
        }
        lds_sync();
        if (kg == 1) return;
        const float m = fmaxf(m_run, at[0]), own = __builtin_amdgcn_exp2f(m_run - m), other = __builtin_amdgcn_exp2f(at[0] - m);
        m_run = m;
        l_run = l_run * own + at[64] * other;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[db][i] = acc[db][i] * own + at[(2 + db * 16 + i) * 64] * other;
    }
    const float sum = l_run + __shfl_xor(l_run, 32, 64);
    if (wave0 + col >= n_items) return;
    // a lane's values: d = 32 db + 8 j + 4 half + r
    if (p.parts > 1) {
        float *rec = p.records + (((size_t)row * a.n_q_heads + head) * p.parts + part) * (REC_HEAD + HD);
        if (half == 0) *reinterpret_cast<float2 *>(rec) = float2{m_run, sum};
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<floatx4 *>(rec + REC_HEAD + db * 32 + j * 8 + half * 4) =
                    floatx4{acc[db][j * 4], acc[db][j * 4 + 1], acc[db][j * 4 + 2], acc[db][j * 4 + 3]};
        return;
    }
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    T *out = (T *)p.out + row * a.out_stride + head * HD + half * 4;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            typedef T four __attribute__((ext_vector_type(4)));
            four x;
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = from_f32<T>(acc[db][j * 4 + r] * inv);
            *reinterpret_cast<four *>(out + db * 32 + j * 8) = x;
        }
}

// Few items (single tokens, drafts, short prompts): a workgroup takes 16 items of one sequence and key head over
// one part of the keys, its four or eight wavefronts the part's tiles of 32 keys in turn, straight from memory into registers: every K and V
// fragment of the pool is one contiguous kilobyte.  The wavefronts' sums meet in LDS.
// Bound by bytes where there are enough sequences (32 tokens behind up to 8191 at 3B: 117 us = 5.0 TB/s, where a copy reaches 4.8; 64
// behind up to 1999 at 1.5B 18.6 us = 3.8 TB/s), else by the launch and four dependent reads (lengths, page ids, keys, values): one token
// behind 1023 at 0.5B 6.1 us, sixteen behind up to 4095 at 1.5B in parts 8.2 us and 3 to 4 for the merge (2.6 TB/s in all).
// 16 items leave half of a 16x16 product empty for groups of 6 to 8 heads, which costs nothing here; 32 a workgroup were no faster.
// Operands of a 16x16 product over 32 values of k: 16 lanes each take 8.
__device__ __forceinline__ floatx4 mma16(const Frag<bf16_t> &a, const Frag<bf16_t> &b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ floatx4 mma16(const Frag<float> &a, const Frag<float> &b, floatx4 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[j], b.v[j], c, 0, 0, 0);
    return c;
}
template <typename T> __device__ __forceinline__ Frag<T> load_frag(const char *at) {
    Frag<T> f;
    const Eight<T> x = *reinterpret_cast<const Eight<T> *>(at);
#pragma unroll
    for (int j = 0; j < 8; ++j) f.v[j] = x.v[j];
    return f;
}

template <typename T, int HD, int WAVES>
__global__ __launch_bounds__(WAVES * 64) VF_MFMA_KERNEL void attention_few_kernel(PackedAttn p) {
    constexpr int KD = HD / 32, DB = HD / 16, FRAG = 512 * (int)sizeof(T), BM = FEW_ITEMS, OUT = HD + 4;   // FRAG: bytes; OUT: stride of a sum in LDS
    extern __shared__ __align__(16) float sums[];   // [WAVES][BM][OUT], then maxima and sums of weights
    float *maxima = sums + WAVES * BM * OUT, *totals = maxima + WAVES * BM;
    const vf_packed_args &a = p.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g4 = lane >> 4, l15 = lane & 15;
    const int rest = p.by_heads(blockIdx.x), kvh = blockIdx.x - rest * a.n_kv_heads, part = p.by_tiles(rest), place = rest - part * p.tiles;
    const int p_first = part * p.part_pages;
    Tile t = {place, 0, 0, 0, 0};
    int ids;   // of the part's first 64 pages, one per lane
    if (p.tile_is_seq) {   // all items of a sequence, a tile after the other (mostly there is one)
        ids = p.table[(size_t)place * a.table_stride + min(p_first + lane, a.max_pages - 1)];   // asked for with the lengths
        const int2 r = seq_rows(p, place);
        t.row0 = __builtin_amdgcn_readfirstlane(r.x);
        t.rows = __builtin_amdgcn_readfirstlane(r.y);
        t.kv_len = __builtin_amdgcn_readfirstlane(seq_keys(p, place));
    } else {
        t = find_tile<BM>(p, place, false);
        ids = p.table[(size_t)t.seq * a.table_stride + min(p_first + lane, a.max_pages - 1)];
    }
    const int32_t *table = p.table + (size_t)t.seq * a.table_stride;
    const int row0 = t.row0, rows = t.rows, kv_len = t.kv_len;
    const int group = p.group, n_items = rows * group, cap = min(kv_len, a.max_pages * VF_TILE), first_pos = kv_len - rows;
    const size_t page_bytes = (size_t)2 * a.n_kv_heads * VF_TILE * HD * sizeof(T), head_bytes = (size_t)VF_TILE * HD * sizeof(T);
    const int items_end = p.tile_is_seq ? n_items : min(n_items, t.item0 + BM);
    for (int item0 = t.item0; item0 < items_end; item0 += BM) {
        const int last = min(first_pos + p.by_group(min(n_items - 1, item0 + BM - 1)), cap - 1);   // last key that an item sees
        const int pages = last < 0 ? 0 : last / VF_TILE + 1, parts = min(p.parts, (pages + p.part_pages - 1) / p.part_pages);
        const int p_end = part == p.parts - 1 ? pages : min(pages, p_first + p.part_pages);
        if (p.parts > 1 && part == 0 && kvh == 0 && threadIdx.x < BM && item0 + (int)threadIdx.x < n_items) {
            // Of a row whose heads lie in two tiles the first tile tells: the second has as many parts or more, of which the
            // row sees no key past the first's, and which the heads of the first have no records of.
            const int at = item0 + threadIdx.x, of = p.by_group(at);
            if (at == of * group) p.used[row0 + of] = parts;
        }
        if (p_first >= p_end && part > 0) continue;
        Frag<T> qf[KD];
        const int item = min(n_items - 1, item0 + l15), item_row = p.by_group(item), last_key = min(first_pos + item_row, cap - 1);
        const T *q = (const T *)p.q + (row0 + item_row) * a.q_stride + (kvh * group + item - item_row * group) * HD + g4 * 8;
#pragma unroll
        for (int kd = 0; kd < KD; ++kd) qf[kd] = load_frag<T>((const char *)(q + kd * 32));
        floatx4 acc[DB];
        float m_run = LOWEST, l_run = 0.f, by = p.scale_log2e;   // by, far: see attention_tiles_kernel
        bool far = false;
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db] = floatx4{0.f, 0.f, 0.f, 0.f};
        // keys 32 i .. + 31, i = 2 p_first + wave, + WAVES ..
        const int first_all = min(first_pos + p.by_group(item0), cap - 1);   // last key that all items see
        const int i_end = min(2 * p_end, last / 32 + 1);
        int ids_at = p_first;   // (a second tile starts over)
        if (item0 != t.item0) ids = table[min(p_first + lane, a.max_pages - 1)];
        Frag<T> k[2 * KD], v[DB];   // a tile's keys are asked for when those before have been multiplied, its values likewise
        auto page = [&](int i) {    // page id of tile i, -1: not in the pool
            const int pg = i / 2;
            if (pg - ids_at >= 64) {
                ids_at = pg;
                ids = table[min(pg + lane, a.max_pages - 1)];
            }
            const int id = __builtin_amdgcn_readlane(ids, pg - ids_at);
            return (unsigned)id < (unsigned)a.pool_pages ? id : -1;
        };
        const char *kv = (const char *)p.kv + kvh * head_bytes + lane * 8 * sizeof(T);
        auto load_k = [&](int i, int id) {
            const char *at = kv + (size_t)max(id, 0) * page_bytes + (i & 1) * (KD * 2 * FRAG);
#pragma unroll
            for (int f = 0; f < 2 * KD; ++f) k[f] = load_frag<T>(at + f * FRAG);
        };
        auto load_v = [&](int i, int id) {
            const char *at = kv + (size_t)max(id, 0) * page_bytes + a.n_kv_heads * head_bytes + (i & 1) * (DB * FRAG);
#pragma unroll
            for (int f = 0; f < DB; ++f) v[f] = load_frag<T>(at + f * FRAG);
        };
        int id = -1;
        if (2 * p_first + wave < i_end) {
            id = page(2 * p_first + wave);
            load_k(2 * p_first + wave, id);
            load_v(2 * p_first + wave, id);
        }
        for (int i = 2 * p_first + wave, id_next; i < i_end; i += WAVES, id = id_next) {
            const int i_next = min(i + WAVES, i_end - 1);   // past the end: the last tile again, not used
            id_next = page(i_next);
            const int own = i * 32 + g4 * 8;                // key of score j: own + j
            const bool masked = i * 32 + 31 > first_all;
            float s[8];
            floatx4 c[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int kd = 0; kd < KD; ++kd)
#pragma unroll
                for (int h = 0; h < 2; ++h) c[h] = mma16(k[h * KD + kd], qf[kd], c[h]);
            float mx = -INFINITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                s[j] = id < 0 || (masked && own + j > last_key) ? -INFINITY : c[j >> 2][j & 3];
                mx = fmaxf(mx, s[j]);
            }
            mx *= p.scale_log2e;
            if (__builtin_amdgcn_ballot_w64(mx > m_run + 8.f)) {   // with slack: see attention_tiles_kernel
                mx = over_item(mx, [](float u, float v) { return fmaxf(u, v); });
                const float m_new = fmaxf(m_run, mx), keep = __builtin_amdgcn_exp2f(m_run - m_new);
                l_run *= keep;
#pragma unroll
                for (int db = 0; db < DB; ++db) acc[db] *= keep;
                m_run = m_new;
                far = __builtin_amdgcn_ballot_w64(fabsf(m_new) > 0x1p24f && m_new != LOWEST);
                by = far ? 1.f : p.scale_log2e;
            }
            if (far) {
#pragma clang fp contract(off)
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] *= p.scale_log2e;
            }
            load_k(i_next, id_next);
            // values of keys that nobody sees count as zeros; one that only some items see and that is not finite would reach
            // the others as 0 times it: then each row takes the product with its own keys
            bool bad = false;
            if (masked || id < 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int db = 0; db < DB; ++db) {
                        if (id < 0 || own + j > last) v[db].v[j] = from_f32<T>(0.f);
                        bad |= own + j > first_all && not_finite(to_f32(v[db].v[j]));
                    }
            }
            // bfloat16 weights as a sum of two (16 significant bits): the loads, not the products, are what this kernel waits for.
            // The first is rounded towards zero and the second never zero beside it, so that an infinite value stays one.
            Frag<T> hi, lo;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float w = __builtin_amdgcn_exp2f(fmaf(s[j], by, -m_run));
                l_run += w;
                if constexpr (sizeof(T) == 2) {
                    const float top = __uint_as_float(__float_as_uint(w) & 0xffff0000u);
                    hi.v[j] = from_f32<T>(top);
                    lo.v[j] = from_f32<T>(fmaxf(w - top, w * 0x1p-24f));
                } else {
                    hi.v[j] = w;
                }
            }
            auto product = [&](const Frag<T> &x, floatx4 sum) {
                sum = mma16(x, hi, sum);
                if constexpr (sizeof(T) == 2) sum = mma16(x, lo, sum);
                return sum;
            };
            if (!__builtin_amdgcn_ballot_w64(bad)) {
#pragma unroll
                for (int db = 0; db < DB; ++db) acc[db] = product(v[db], acc[db]);
            } else {
                static_for<0, DB>([&](auto db) {
                    constexpr int D = db;
                    floatx4 sum = acc[D];
                    for (int seen = max(first_all, i * 32); seen <= min(last, i * 32 + 31); ++seen) {
                        Frag<T> x = v[D];
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (own + j > seen) x.v[j] = from_f32<T>(0.f);
                        const floatx4 of_row = product(x, acc[D]);
                        if (min(last_key, i * 32 + 31) == seen) sum = of_row;
                    }
                    acc[D] = sum;
                    __builtin_amdgcn_sched_barrier(0);   // one block's values in registers at a time
                });
            }
            load_v(i_next, id_next);
        }
        // sums of the wavefronts; a lane's values: item l15, d = 16 db + 4 g4 + r
        if (item0 != t.item0) __syncthreads();
        const float l = over_item(l_run, [](float u, float v) { return u + v; });
        const int at = wave * BM + l15;
        if (g4 == 0) { maxima[at] = m_run; totals[at] = l; }
#pragma unroll
        for (int db = 0; db < DB; ++db) *reinterpret_cast<floatx4 *>(&sums[at * OUT + db * 16 + g4 * 4]) = acc[db];
        __syncthreads();
        for (int j = threadIdx.x; j < BM * (HD / 4); j += WAVES * 64) {
            const int it = j / (HD / 4), d0 = j % (HD / 4) * 4, item = item0 + it;
            if (item >= n_items) break;
            float M = LOWEST, L = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) M = fmaxf(M, maxima[w * BM + it]);
            floatx4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = __builtin_amdgcn_exp2f(maxima[w * BM + it] - M);
                L += totals[w * BM + it] * f;
                o += *reinterpret_cast<const floatx4 *>(&sums[(w * BM + it) * OUT + d0]) * f;
            }
            const int item_row = p.by_group(item), row = row0 + item_row, head = kvh * group + item - item_row * group;
            if (p.parts > 1) {
                float *rec = p.records + (((size_t)row * a.n_q_heads + head) * p.parts + part) * (REC_HEAD + HD);
                if (d0 == 0) *reinterpret_cast<float2 *>(rec) = float2{M, L};
                *reinterpret_cast<floatx4 *>(rec + REC_HEAD + d0) = o;
            } else {
                const float inv = L == 0.f ? 0.f : 1.0f / L;
                typedef T four __attribute__((ext_vector_type(4)));
                four x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = from_f32<T>(o[e] * inv);
                *reinterpret_cast<four *>((T *)p.out + row * a.out_stride + head * HD + d0) = x;
            }
        }
    }
}

// Merge of the parts: HD / 4 threads per row and head.  Three dependent reads and a launch: 2.8 to 4 us.
template <typename T, int HD>
__global__ __launch_bounds__(256) void attention_merge_kernel(PackedAttn p) {
    constexpr int REC = HD + REC_HEAD, TH = HD / 4;
    const vf_packed_args &a = p.a;
    const int idx = blockIdx.x * (256 / TH) + threadIdx.x / TH;
    const int row = p.by_q_heads(idx), head = idx - row * a.n_q_heads, d0 = threadIdx.x % TH * 4;
    if (row >= a.total_rows) return;
    const bool inside = row >= p.row_off[0] && row < p.row_off[a.n_seqs];
    const float *rec = p.records + ((size_t)row * a.n_q_heads + head) * p.parts * REC;
    float M = LOWEST, L = 0.f;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    // NR records are asked for together; how many there are is read first (asked for with all of a row's records, which spares
    // a round trip, many rows took up to a quarter longer for records that are not there, and few no less)
    constexpr int NR = 8;
    const int used = min(p.parts, p.used[row]);
    for (int i0 = 0; i0 < used; i0 += NR) {
        float2 ml[NR];
        floatx4 v[NR];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const float *r = rec + (size_t)min(i0 + i, used - 1) * REC;
            ml[i] = *reinterpret_cast<const float2 *>(r);
            v[i] = *reinterpret_cast<const floatx4 *>(r + REC_HEAD + d0);
        }
        float m = M;
#pragma unroll
        for (int i = 0; i < NR; ++i)
            if (i0 + i < used) m = fmaxf(m, ml[i].x);
        const float keep = __builtin_amdgcn_exp2f(M - m);
        L *= keep;
        acc *= keep;
        M = m;
#pragma unroll
        for (int i = 0; i < NR; ++i)
            if (i0 + i < used) {
                const float add = __builtin_amdgcn_exp2f(ml[i].x - m);
                L += ml[i].y * add;
                acc += v[i] * add;
            }
    }
    if (!inside) return;
    const float inv = L == 0.f ? 0.f : 1.0f / L;
    typedef T four __attribute__((ext_vector_type(4)));
    four x;
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = from_f32<T>(acc[r] * inv);
    *reinterpret_cast<four *>((T *)p.out + row * a.out_stride + head * HD + d0) = x;
}

int check(const char *name, const vf_packed_args *args) {
    if (!args) return vf_fail(VF_ERR_ARG, "%s: NULL argument", name);
    const vf_packed_args &a = *args;
    if (a.dtype != VF_F32 && a.dtype != VF_BF16) return vf_fail(VF_ERR_ARG, "%s: dtype %d", name, a.dtype);
    if (a.n_q_heads < 1 || a.n_kv_heads < 1 || a.n_q_heads > 256 || a.n_q_heads % a.n_kv_heads)
        return vf_fail(VF_ERR_ARG, "%s: %d query heads, %d key heads", name, a.n_q_heads, a.n_kv_heads);
    if (a.head_dim != 64 && a.head_dim != 128) return vf_fail(VF_ERR_UNSUPPORTED, "%s: head_dim %d (built for 64 and 128)", name, a.head_dim);
    if (a.n_seqs < 1 || a.n_seqs > VF_PACKED_MAX_SEQS || a.total_rows < 0 || a.total_rows > VF_PACKED_MAX_ROWS)
        return vf_fail(VF_ERR_ARG, "%s: %d sequences, %d rows", name, a.n_seqs, a.total_rows);
    if (a.max_rows < 0 || a.max_keys < 0 || a.pool_pages < 1 || a.pool_pages > 0x7fffffff / VF_TILE || a.max_pages < 1 ||
        a.max_pages > 0x7fffffff / VF_TILE || a.table_stride < a.max_pages)
        return vf_fail(VF_ERR_ARG, "%s: max_rows %d, max_keys %d, pool_pages %d, max_pages %d, table_stride %d", name, a.max_rows,
                       a.max_keys, a.pool_pages, a.max_pages, a.table_stride);
    if (!std::isfinite(a.scale) || a.scale < 0) return vf_fail(VF_ERR_ARG, "%s: scale %g", name, a.scale);
    const int64_t w = (int64_t)a.n_q_heads * a.head_dim;
    if (a.q_stride < w || a.out_stride < w)
        return vf_fail(VF_ERR_ARG, "%s: rows overlap (strides %lld, %lld)", name, (long long)a.q_stride, (long long)a.out_stride);
    if ((a.q_stride | a.out_stride) * (a.dtype == VF_BF16 ? 2 : 4) & 15)
        return vf_fail(VF_ERR_UNSUPPORTED, "%s: strides are multiples of 16 bytes", name);
    return VF_OK;
}

// ---- choice of kernel and parts -------------------------------------------------------------------

enum { TILES = 0, TILES_TWO = 1, FEW = 2, N_KERNELS = 3 };   // 128 items a workgroup; the same, two groups of wavefronts; 16 items
constexpr int MAX_WORKGROUPS = 0x7fffff;   // of 512 threads, whose number stays below 2^32; tiles of 128 items and no parts never have more
struct Plan { int kernel, tile_is_seq, tiles, parts, part_pages, waves; size_t bytes; };

// What a call costs, in us: the way of the longest workgroup through its pages or the chip's way through all of them, whichever is
// longer, and a merge.  The constants are fits to 191 calls (prompts, chunks behind a prefix, drafts and single
// tokens of 1 to 64 sequences in four shapes, with every kernel and the numbers of parts below:
// profiles/packed_attention_plan_timings.txt); the choice costs 0.9 % on average against the best of all (tiles of 128 items
// without parts throughout: 223 %), 13 % at most.  What the kernels are to one another, in us: 2048 tokens at 1.5B 38 with 128 items, 33
// with two groups, 57 with 16; six prompts of up to 4096 166, 188, 491; 22 rows behind 2000 in six parts 14.8, 15.6, 10.2, in one 36.8,
// 31.6, 13.9; drafts of 16 sequences in eight parts 25, 22, 41.
struct KernelCost {
    float start, page, page_full;   // the longest way: with up to half as many workgroups as the chip holds, with as many and more
    float load_page, load_start;    // a chip full of workgroups: a page, a workgroup
};
struct TypeCost {
    KernelCost k[N_KERNELS + 1];    // the last: 16 items, four wavefronts
    float merge, merge_mb, merge8;
};
constexpr TypeCost COST[3] = {
    {{{2.991f, 1.12f, 1.167f, 1.143f, 0.001f}, {6.042f, 0.6525f, 0.5752f, 0.4454f, 3.089f}, {1.302f, 0.2779f, 0.3042f, 0.09254f, 1.694f}, {4.439f, 0.4318f, 0.43f, 0.4294f, 0.2164f}}, 5.297f, 0.4362f, 1.178f},   // bfloat16, heads of 64
    {{{4.291f, 0.9058f, 0.7355f, 0.7817f, 1.317f}, {5.425f, 0.8706f, 0.5725f, 0.4849f, 2.104f}, {3.007f, 0.4337f, 0.3039f, 0.281f, 1.466f}, {4.181f, 0.6562f, 0.7576f, 0.5794f, 1.727f}}, 4.363f, 0.6175f, 2.549f},   // bfloat16, heads of 128
    {{{2.321f, 5.142f, 7.635f, 1.674f, 0.5421f}, {/* no two groups */}, {2.393f, 0.691f, 0.4236f, 0.622f, 0.001f}, {8.491f, 0.7689f, 1.807f, 1.221f, 1.31f}}, 4.161f, 1.255f, 0.001072f},   // float32
};

Plan make_plan(const vf_packed_args &a) {
    Plan best{};
    const int cost_of = a.dtype == VF_F32 ? 2 : a.head_dim == 64 ? 0 : 1;
    const TypeCost &cost = COST[cost_of];
    const int group = a.n_q_heads / a.n_kv_heads, seqs = std::min(a.n_seqs, a.total_rows);
    const int pages = std::max(1, std::min(a.max_pages, (int)(((long long)a.max_keys + VF_TILE - 1) / VF_TILE)));
    const long long most_items = (long long)std::min(a.max_rows, a.total_rows) * group, items = (long long)a.total_rows * group;
    // pages that an item sees on average: rows do not see the call's later ones (how much shorter the other sequences are than
    // the longest the host does not say)
    const float whole = std::min(1.f, (float)a.max_rows / std::max(1, a.max_keys));
    const float mean = std::max(1.f, pages * (1.f - 0.5f * whole));
    float best_cost = 0.f;
    for (int kernel = 0; kernel < N_KERNELS; ++kernel) {
        if (kernel == TILES_TWO && a.dtype == VF_F32) continue;   // one wavefront's float32 products fill a matrix unit
        if (kernel != FEW && most_items <= FEW_ITEMS) continue;     // every sequence one tile of 16: bound by memory, and more exact there
        const int bm = kernel == FEW ? FEW_ITEMS : TILE_WAVES * 32;
        const bool tile_is_seq = kernel == FEW && most_items <= bm;
        const long long tiles = tile_is_seq ? a.n_seqs : items / bm + seqs;   // a sequence ends in one tile that is not full
        const float groups = (tile_is_seq ? seqs : items / (float)bm + (seqs > 1 ? 0.5f * seqs : 0.5f)) * a.n_kv_heads;
        for (const int parts : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16}) {
            const int part_pages = (pages + parts - 1) / parts;
            if ((pages + part_pages - 1) / part_pages != parts || tiles * parts * a.n_kv_heads > MAX_WORKGROUPS) continue;
            const float used = parts == 1 ? 1.f : std::min((float)parts, mean / part_pages + 1.f);
            const float workgroups = groups * used;
            // Tiles of 16 items: eight wavefronts share a tile's keys, or four where there are more tiles than compute units, of which one
            // holds two or three such: 512 tokens at 1.5B 8.5 us for 11.8, 256 single tokens at 0.5B 18.7 for 19.9, thousands of tiles
            // 0.6 to 0.8 of the time; one token behind 1023 at 0.5B 7.4 for 6.1.
            const bool four = kernel == FEW && workgroups > 256.f;
            const KernelCost &k = cost.k[four ? N_KERNELS : kernel];
            const int chip = four ? 512 : kernel != TILES ? 256 : cost_of == 0 ? 768 : 512;   // workgroups on 256 compute units
            const float crowd = std::min(1.f, std::max(0.f, 2 * workgroups / chip - 1.f));
            const float way = part_pages * (k.page + (k.page_full - k.page) * crowd), load = workgroups / chip * (k.load_page * mean / used + k.load_start);
            float us = k.start + std::max(way, load);
            if (parts > 1) us += cost.merge + cost.merge_mb * 4e-6f * a.total_rows * a.n_q_heads * used * (REC_HEAD + a.head_dim) + cost.merge8 * (((int)used - 1) / 8);
            // less than the host takes for a call of one launch or two is not gained (one token behind 1024 at 0.5B in three parts 11.1 us, whole 8.0)
            us = std::max(us, parts > 1 ? 10.f : 8.f) + 0.1f * us;
            if (best.parts && us >= best_cost) continue;
            best_cost = us;
            best = {kernel, tile_is_seq, (int)tiles, parts, part_pages, four ? 4 : 8, 0};
        }
    }
    if (best.parts > 1)
        best.bytes = (size_t)a.total_rows * a.n_q_heads * best.parts * (REC_HEAD + a.head_dim) * sizeof(float) + (size_t)a.total_rows * sizeof(int32_t);
    return best;
}

// Workgroups in the order of their numbers: the first parts of all tiles (those that exist for all), then the second .. A die takes every
// eighth workgroup: with the parts of a tile next to one another some dies had the full ones and some the rest
// (a prompt of 4096 tokens at 0.5B in two parts 70 us).
template <typename F> int start(F kernel, long long blocks, int threads, int lds, const PackedAttn &p, hipStream_t st) {
    if (blocks > MAX_WORKGROUPS) return vf_fail(VF_ERR_UNSUPPORTED, "vf_attention_packed: %lld workgroups", blocks);
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads), lds, st, p);
    VF_LAUNCH_CHECK("attention_packed");
    return VF_OK;
}
template <typename T, int HD, int WAVES> int launch_few(const PackedAttn &p, hipStream_t st) {
    constexpr int LDS = WAVES * FEW_ITEMS * (HD + 6) * 4;
    static const hipError_t set = hipFuncSetAttribute((const void *)attention_few_kernel<T, HD, WAVES>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    VF_HIP(set);
    return start(attention_few_kernel<T, HD, WAVES>, (long long)p.tiles * p.parts * p.a.n_kv_heads, WAVES * 64, LDS, p, st);
}
template <typename T, int HD, int KG> int launch_tiles(const PackedAttn &p, hipStream_t st) {
    constexpr int LDS = KG * 2 * HD / 4 * 1024 * (int)sizeof(T) / 2;
    static const hipError_t set = hipFuncSetAttribute((const void *)attention_tiles_kernel<T, HD, KG>, hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    VF_HIP(set);
    return start(attention_tiles_kernel<T, HD, KG>, (long long)p.tiles * p.parts * p.a.n_kv_heads, TILE_WAVES * KG * 64, LDS, p, st);
}
template <typename T, int HD> int launch_kernel(const PackedAttn &p, const Plan &plan, hipStream_t st) {
    if (plan.kernel == FEW) return plan.waves == 4 ? launch_few<T, HD, 4>(p, st) : launch_few<T, HD, 8>(p, st);
    if constexpr (sizeof(T) == 2)
        if (plan.kernel == TILES_TWO) return launch_tiles<T, HD, 2>(p, st);
    return launch_tiles<T, HD, 1>(p, st);
}
template <typename T, int HD> int launch(const PackedAttn &p, const Plan &plan, hipStream_t st) {
    const int rc = launch_kernel<T, HD>(p, plan, st);
    if (rc != VF_OK || p.parts == 1) return rc;
    constexpr int PER = 256 / (HD / 4);
    return start(attention_merge_kernel<T, HD>, ((long long)p.a.total_rows * p.a.n_q_heads + PER - 1) / PER, 256, 0, p, st);
}

}  // namespace

extern "C" {

// Which kernel and how many parts a call takes: for the test that holds the choice against kept timings.
int vf_debug_packed_plan(const vf_packed_args *args, int *kernel, int *parts) {
    if (const int rc = check("vf_debug_packed_plan", args)) return rc;
    const Plan plan = make_plan(*args);
    *kernel = plan.kernel;
    *parts = plan.parts;
    return VF_OK;
}

size_t vf_attention_packed_workspace(const vf_packed_args *args) {
    if (check("vf_attention_packed_workspace", args) != VF_OK) return (size_t)-1;
    return make_plan(*args).bytes;
}

int vf_attention_packed(const vf_packed_args *args, const void *q_dev, const void *kv_layer_dev, const int32_t *block_table_dev,
                        const int32_t *row_off_dev, const int32_t *kv_len_dev, void *out_dev, void *workspace_dev, size_t workspace_bytes,
                        void *stream) {
    if (int rc = check("vf_attention_packed", args)) return rc;
    PackedAttn p = {};
    p.a = *args;
    if (p.a.total_rows == 0) return VF_OK;
    if (!q_dev || !kv_layer_dev || !block_table_dev || !row_off_dev || !kv_len_dev || !out_dev)
        return vf_fail(VF_ERR_ARG, "vf_attention_packed: NULL argument");
    if (((uintptr_t)q_dev | (uintptr_t)kv_layer_dev | (uintptr_t)out_dev | (uintptr_t)workspace_dev) & 15)
        return vf_fail(VF_ERR_UNSUPPORTED, "vf_attention_packed: addresses are multiples of 16 bytes");
    const Plan plan = make_plan(p.a);
    if (plan.bytes && !workspace_dev) return vf_fail(VF_ERR_ARG, "vf_attention_packed: needs a workspace of %zu bytes", plan.bytes);
    if (plan.bytes > workspace_bytes) return vf_fail(VF_ERR_CAP, "vf_attention_packed: workspace of %zu bytes, needs %zu", workspace_bytes, plan.bytes);
    p.q = q_dev;
    p.kv = kv_layer_dev;
    p.table = block_table_dev;
    p.row_off = row_off_dev;
    p.kv_len = kv_len_dev;
    p.out = out_dev;
    p.group = p.a.n_q_heads / p.a.n_kv_heads;
    p.tiles = plan.tiles;
    p.tile_is_seq = plan.tile_is_seq;
    p.parts = plan.parts;
    // Where workgroups meet on a CU, or wait for one, the long ones go first: twelve prompts of 230 to 2048 tokens at 0.5B 73 -> 69 us,
    // six of 451 to 4096 at 1.5B 177 -> 169 us.  The search costs a workgroup up to 2 us (drafts of 16 sequences in parts,
    // 276 workgroups: 23.5 -> 25.8 us), so calls that are split or have a workgroup a CU take the sequences as they come.
    p.by_height = plan.kernel != FEW && plan.parts == 1 && p.a.n_seqs > 1 && (long long)plan.tiles * p.a.n_kv_heads > 256;
    p.part_pages = plan.part_pages;
    p.scale_log2e = (p.a.scale == 0.f ? 1.0f / sqrtf((float)p.a.head_dim) : p.a.scale) * 1.4426950408889634f;
    p.by_group = divisor(p.group);
    p.by_heads = divisor(p.a.n_kv_heads);
    p.by_tiles = divisor(plan.tiles);
    p.by_q_heads = divisor(p.a.n_q_heads);
    p.records = (float *)workspace_dev;
    p.used = (int32_t *)((char *)workspace_dev + plan.bytes - (size_t)p.a.total_rows * sizeof(int32_t));
    const auto go = p.a.dtype == VF_BF16 ? (p.a.head_dim == 128 ? launch<bf16_t, 128> : launch<bf16_t, 64>)
                                         : (p.a.head_dim == 128 ? launch<float, 128> : launch<float, 64>);
    return go(p, plan, (hipStream_t)stream);
}

}  // extern "C"
