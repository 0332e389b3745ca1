// Penalties for repeated tokens, biases and grammar masks on the logits of packed rows.
#include <algorithm>
#include <type_traits>

#include "vf_internal.h"

namespace {

struct LogitsArrays {
    const int32_t *row_off;
    const float *penalties;                                // [n_seqs][3] or NULL
    const int32_t *history, *history_len, *prompt_len;     // NULL: none; prompt_len NULL: no prompt
    const int32_t *tokens;                                 // [total_rows] or NULL
    const int32_t *bias_off, *bias_id;                     // NULL: none
    const float *bias;
    const uint32_t *mask;                                  // [mask_rows][mask_stride] or NULL
    const int32_t *mask_row;                               // [total_rows]; NULL: row r has mask r
};

constexpr int LOGIT_THREADS = 256;

// The sequence that has row `row`: the number of offsets that are not above it, less one.
__device__ __forceinline__ int sequence_of(const int32_t *__restrict__ row_off, int n_seqs, int row) {
    const int lane = threadIdx.x & 63;
    int not_above = 0;
    for (int i0 = lane; i0 - lane <= n_seqs; i0 += 256) {
        int off[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) off[j] = row_off[min(i0 + j * 64, n_seqs)];
#pragma unroll
        for (int j = 0; j < 4; ++j) not_above += __popcll(__ballot(i0 + j * 64 <= n_seqs && off[j] <= row));
    }
    return not_above - 1;
}

// A value that is the same for the whole wavefront, through the scalar cache (nobody writes what a call reads): vector loads come back in the
// order in which they were asked for, so this one does not wait for the logits that are on their way.
template <typename T> __device__ __forceinline__ T uniform(const T *p, int i) {
    return reinterpret_cast<const __attribute__((address_space(4))) T *>(reinterpret_cast<uintptr_t>(p))[i];
}

// Keeps the compiler from putting off such reads to where each is used first, so that they are on their way together.
__device__ __forceinline__ void together(int a, int b, int c, int d, float e, float f, float g) {
    asm volatile("" : : "s"(a), "s"(b), "s"(c), "s"(d), "s"(e), "s"(f), "s"(g));
}

// Loads and stores of a row's piece through a buffer descriptor: one 32-bit offset a lane, and what lies past the piece's end is read as 0
// and not written, so that no access has a condition of its own.
typedef unsigned uint4v __attribute__((ext_vector_type(4)));
__device__ __forceinline__ __amdgpu_buffer_rsrc_t piece(const void *start, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(start), 0, bytes, 0x00027000);
}
template <typename T, int N> struct alignas(N * sizeof(T)) Some { T v[N]; };
template <typename T, int N> __device__ __forceinline__ Some<T, N> read_some(__amdgpu_buffer_rsrc_t p, int element) {
    constexpr int BYTES = N * sizeof(T);
    const int at = element * (int)sizeof(T);
    if constexpr (BYTES == 16) return __builtin_bit_cast(Some<T, N>, __builtin_amdgcn_raw_buffer_load_b128(p, at, 0, 0));
    else if constexpr (BYTES == 8) return __builtin_bit_cast(Some<T, N>, __builtin_amdgcn_raw_buffer_load_b64(p, at, 0, 0));
    else if constexpr (BYTES == 4) return __builtin_bit_cast(Some<T, N>, __builtin_amdgcn_raw_buffer_load_b32(p, at, 0, 0));
    else return __builtin_bit_cast(Some<T, N>, __builtin_amdgcn_raw_buffer_load_b16(p, at, 0, 0));
}
// How a call writes: through the caches, past them, or over the logits themselves, where only what changes is read and written.
enum Way { CACHED, PAST, IN_PLACE };
template <int N, Way WAY> __device__ __forceinline__ void write_some(__amdgpu_buffer_rsrc_t p, int element, const Some<float, N> &x) {
    constexpr int NT = WAY == PAST ? 2 : 0;
    if constexpr (N == 4) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uint4v, x), p, element * 4, 0, NT);
    else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, x), p, element * 4, 0, NT);
}

struct Penalty { float repetition, presence, frequency, scale, divisor, inverse; };   // divisor = repetition * scale, inverse = 1 / divisor

// z with the penalties of an id that the text has.  count: bit 0: seen in the prompt; above: how often given.  The quotient is that by the
// reciprocal with one correction (its remainder is exact), which is a few instructions where a division is ten.  A repetition that has no
// reciprocal in the type is scaled to one that has, and the logit with it (17 rows of 151,936 ids 8.6 us in a graph, with a division for all 8.8).
__device__ __forceinline__ float penalised(float z, unsigned count, const Penalty &p) {
    const float x = z * p.scale, q = x * p.inverse, quotient = fmaf(fmaf(-q, p.divisor, x), p.inverse, q);
    z = z > 0.f ? (q < INFINITY ? quotient : q) : z * p.repetition;
    if (count >> 1) z -= p.presence + p.frequency * (float)(count >> 1);
    return z;
}

// A workgroup has SLICE ids of some rows.  Two tables in LDS hold how often the sequence's text has each id and its bias; they are made
// once for the rows of a sequence, and a row adds its own token.  Counts are whole numbers, so the order of the additions does not
// matter, and of several biases of an id the last of the list is found as a maximum over their places.
//
// It is bound by memory, and for few rows by reads that wait for one another: all that depends on the sequence alone is asked for with its offsets,
// for a sequence that is guessed (right where all have as many rows), then come the text, biases and masks, and the tables.  What the
// tables cost is time in which a workgroup's loads and stores rest: 70 rows of 128,256 bfloat16 logits with texts of 1500 and 300 biases each take
// 18.2 us in a graph (3.0 TB/s), about 13 without the tables; seven workgroups a compute unit hide the rest of it.  One row of
// 151,936 ids 3.9 us, 270 rows of 16 sequences with everything 66.0 us (5.05 TB/s; a large copy 4.74).
// Over themselves 170 rows with texts of 2000 and 40 biases take 31.9 us, apart 33.8, though without masks only 37 MB are read and 11 written where apart
// 103 go each way: the same slices find the few ids that change, and each reads the whole text.
// Rows that do not start at a multiple of four ids keep fewer tokens in flight, for eight wavefronts a SIMD: 100 rows of 100,003 ids 24.4 us for 26.5.
template <typename T, int SLICE, bool VEC, Way WAY>
__global__ __launch_bounds__(LOGIT_THREADS, VEC ? 1 : 8) void logits_adjust_kernel(vf_logits_args a, LogitsArrays x, const T *logits, float *out, int slices,
                                                                      int rows_each) {
    constexpr int EACH = SLICE / LOGIT_THREADS, STEP = VEC ? 4 : 1, TEXT = VEC ? 8 : 4, BIASES = 2;   // ids a thread, how many side by side, tokens and
                                                                                              // biases asked for at a time
    __shared__ __align__(16) unsigned count[SLICE], bias[SLICE];     // (bias: the bits of a float)
    const int tid = threadIdx.x, chunk = blockIdx.x / slices, v0 = (blockIdx.x - chunk * slices) * SLICE;
    const int r0 = chunk * rows_each, r1 = (int)min((long long)r0 + rows_each, (long long)a.total_rows);
    const int ids = min(SLICE, a.vocab - v0);
    // a thread's ids: four in a row EACH / 4 times, or LOGIT_THREADS apart
    auto id_of = [&](int i) { return i * (STEP * LOGIT_THREADS) + tid * STEP; };
    for (int i = tid; i < SLICE; i += LOGIT_THREADS) {
        count[i] = 0;
        bias[i] = 0;
    }
    // the tables' sequence, or a guess at the first row's: right where all have as many rows
    int seq = (int)((long long)r0 * a.n_seqs / a.total_rows), end = 0;
    bool counted = false, biased = false, inside = false, clean = true;
    Penalty p{1.f, 0.f, 0.f, 1.f, 1.f, 1.f};
    for (int r = r0; r < r1; ++r) {
        Some<T, STEP> z[EACH / STEP];
        uint32_t bits[EACH / STEP];
        const auto from = piece(logits + (size_t)r * a.in_stride + v0, ids * (int)sizeof(T));
        const int m = x.mask ? (x.mask_row ? uniform(x.mask_row, r) : r) : -1, own = x.tokens ? uniform(x.tokens, r) : -1;
        const bool masked = m >= 0 && m < a.mask_rows;
        // over itself, a row without a mask changes in few places, which are read when they are known
        const bool whole = WAY != IN_PLACE || masked;
        if (whole)
#pragma unroll
            for (int i = 0; i < EACH / STEP; ++i) z[i] = read_some<T, STEP>(from, id_of(i));
#pragma unroll
        for (int i = 0; i < EACH / STEP; ++i) bits[i] = 0xffffffffu;
        if (masked) {
            const auto words = piece(x.mask + (size_t)m * a.mask_stride + v0 / 32, (ids + 31) / 32 * 4);
#pragma unroll
            for (int i = 0; i < EACH / STEP; ++i) bits[i] = read_some<uint32_t, 1>(words, id_of(i) / 32).v[0];
        }
        if (r >= end) {        // the first row, or the first of another sequence
            int first, length, prompt, b0, b1;
            if (r > r0) seq = min(seq + 1, a.n_seqs - 1);
            for (bool sure = false;; sure = true) {
                // all that depends on the sequence alone is asked for with its offsets, without conditions, whose ends would wait for it: what
                // is not there is read from the offsets instead, and not used
                const float *penalties = x.penalties ? x.penalties + 3 * (size_t)seq : reinterpret_cast<const float *>(x.row_off);
                const int32_t *biases = x.bias_off ? x.bias_off + seq : x.row_off;
                first = uniform(x.row_off, seq);
                end = uniform(x.row_off, seq + 1);
                p = Penalty{uniform(penalties, 0), uniform(penalties, 1), uniform(penalties, x.penalties ? 2 : 1), 0.f, 0.f, 0.f};
                length = uniform(x.history ? x.history_len : x.row_off, seq);
                prompt = uniform(x.prompt_len ? x.prompt_len : x.row_off, seq);
                b0 = uniform(biases, 0);
                b1 = uniform(biases, 1);
                together(length, prompt, b0, b1, p.repetition, p.presence, p.frequency);
                inside = first >= 0 && first <= r && r < end;
                if (sure || inside) break;
                seq = sequence_of(x.row_off, a.n_seqs, r);
                if (seq < 0 || seq >= a.n_seqs) {     // in front of the sequences' rows, or behind them
                    end = seq < 0 ? uniform(x.row_off, 0) : a.total_rows;
                    seq = max(0, min(seq, a.n_seqs - 1));
                    break;
                }
            }
            end = max(end, r + 1);
            if (inside) {
                counted = x.penalties && (p.repetition != 1.f || p.presence != 0.f || p.frequency != 0.f);
                // by infinity: 0 / 1; by what is below the normal numbers, whose reciprocal may be infinite: both times 2^64
                p.scale = p.repetition == INFINITY ? 0.f : fabsf(p.repetition) < 0x1p-126f ? 0x1p64f : 1.f;
                p.divisor = p.repetition == INFINITY ? 1.f : p.repetition * p.scale;
                p.inverse = 1.f / p.divisor;
                const int n = x.history ? min(max(length, 0), a.max_history) : 0;
                prompt = x.prompt_len ? min(max(prompt, 0), n) : 0;
                b1 = x.bias_off ? min(max(b1, 0), a.bias_entries) : 0;
                b0 = min(max(b0, 0), b1);       // (a sum with an offset far past the list would be negative)
                biased = b0 < b1;
                const auto text = piece(x.history + (size_t)seq * a.history_stride, n * 4);
                int id[TEXT];
#pragma unroll
                for (int j = 0; j < TEXT; ++j) id[j] = read_some<int, 1>(text, tid + j * LOGIT_THREADS).v[0];
                unsigned bias_id[BIASES];
#pragma unroll
                for (int j = 0; j < BIASES; ++j) bias_id[j] = b0 + tid + j * LOGIT_THREADS < b1 ? x.bias_id[b0 + tid + j * LOGIT_THREADS] : -1;
                __syncthreads();   // the tables are clear, or the rows before have read them
                if (!clean) {
                    for (int i = tid; i < SLICE; i += LOGIT_THREADS) {
                        count[i] = 0;
                        bias[i] = 0;
                    }
                    __syncthreads();
                }
                clean = !counted && !biased;
                if (counted) {
                    for (int i0 = tid; i0 < n; i0 += TEXT * LOGIT_THREADS) {
                        if (i0 != tid)
#pragma unroll
                            for (int j = 0; j < TEXT; ++j) id[j] = read_some<int, 1>(text, i0 + j * LOGIT_THREADS).v[0];
#pragma unroll
                        for (int j = 0; j < TEXT; ++j) {
                            if (i0 - tid + j * LOGIT_THREADS >= n) break;
                            const unsigned d = (unsigned)id[j] - v0;
                            const int i = i0 + j * LOGIT_THREADS;
                            if (d < SLICE && i < n) {
                                if (i < prompt) atomicOr(&count[d], 1u);
                                else atomicAdd(&count[d], 2u);
                            }
                        }
                    }
                    if (x.tokens)
                        for (int i = first + tid; i < r; i += LOGIT_THREADS) {
                            const unsigned d = (unsigned)x.tokens[i] - v0;
                            if (d < SLICE) atomicAdd(&count[d], 2u);
                        }
                }
                if (biased) {      // first the number of an id's last bias, from 1 on
#pragma unroll
                    for (int j = 0; j < BIASES; ++j)
                        if (bias_id[j] - v0 < SLICE) atomicMax(&bias[bias_id[j] - v0], 1u + tid + j * LOGIT_THREADS);
                    for (int i = b0 + tid + BIASES * LOGIT_THREADS; i < b1; i += LOGIT_THREADS)
                        if (const unsigned d = (unsigned)x.bias_id[i] - v0; d < SLICE) atomicMax(&bias[d], 1u + (i - b0));
                }
                if (counted || biased) __syncthreads();
                if (biased) {      // a thread puts the values in the places of its own ids; without a number it reads past the list: 0
                    const auto values = piece(x.bias + b0, (b1 - b0) * 4);
                    unsigned value[EACH];
#pragma unroll
                    for (int i = 0; i < EACH; ++i) value[i] = bias[id_of(i / STEP) + i % STEP];
#pragma unroll
                    for (int i = 0; i < EACH; ++i) value[i] = read_some<unsigned, 1>(values, (int)value[i] - 1).v[0];
#pragma unroll
                    for (int i = 0; i < EACH; ++i) bias[id_of(i / STEP) + i % STEP] = value[i];
                }
            }
        }
        if (inside) {
            if (counted && x.tokens) {
                const unsigned d = (unsigned)own - v0;
                if (d < SLICE) {
                    __syncthreads();     // the rows before have been read
                    if (tid == 0) count[d] += 2;
                    __syncthreads();
                }
            }
            const auto to = piece(out + (size_t)r * a.out_stride + v0, ids * 4);
            constexpr uint32_t ALL = (1u << STEP) - 1;
#pragma unroll
            for (int i = 0; i < EACH / STEP; ++i) bits[i] >>= id_of(i) % 32;
            bool touched[EACH / STEP];
            if constexpr (WAY == IN_PLACE) {
#pragma unroll
                for (int i = 0; i < EACH / STEP; ++i) {
                    unsigned any = 0;
                    if (counted) {
                        const Some<unsigned, STEP> c = *reinterpret_cast<const Some<unsigned, STEP> *>(count + id_of(i));
#pragma unroll
                        for (int j = 0; j < STEP; ++j) any |= c.v[j];
                    }
                    if (biased) {
                        const Some<unsigned, STEP> b = *reinterpret_cast<const Some<unsigned, STEP> *>(bias + id_of(i));
#pragma unroll
                        for (int j = 0; j < STEP; ++j) any |= b.v[j];
                    }
                    touched[i] = any || (bits[i] & ALL) != ALL;
                    if (!whole) z[i] = any ? read_some<T, STEP>(from, id_of(i)) : Some<T, STEP>{};
                }
            }
#pragma unroll
            for (int i = 0; i < EACH / STEP; ++i) {
                Some<float, STEP> y;
#pragma unroll
                for (int j = 0; j < STEP; ++j) y.v[j] = to_f32(z[i].v[j]);
                if (counted) {
                    const Some<unsigned, STEP> c = *reinterpret_cast<const Some<unsigned, STEP> *>(count + id_of(i));
                    unsigned any = 0;
#pragma unroll
                    for (int j = 0; j < STEP; ++j) any |= c.v[j];
                    if (any) {
#pragma unroll
                        for (int j = 0; j < STEP; ++j)
                            if (c.v[j]) y.v[j] = penalised(y.v[j], c.v[j], p);
                    }
                }
                if (biased) {
                    const Some<unsigned, STEP> b = *reinterpret_cast<const Some<unsigned, STEP> *>(bias + id_of(i));
#pragma unroll
                    for (int j = 0; j < STEP; ++j) y.v[j] += __uint_as_float(b.v[j]);
                }
#pragma unroll
                for (int j = 0; j < STEP; ++j) y.v[j] = bits[i] >> j & 1 ? y.v[j] : -INFINITY;
                if (WAY != IN_PLACE || touched[i]) write_some<STEP, WAY>(to, id_of(i), y);
            }
        }
    }
}

template <typename T, int SLICE, bool VEC, Way WAY>
int launch_slices(const vf_logits_args &a, const LogitsArrays &x, const void *logits, float *out, hipStream_t st) {
    const int slices = (a.vocab + SLICE - 1) / SLICE;
    // rows that are likely to be of one sequence share its tables, up to three and as long as about 600 workgroups are left (136 rows of 8
    // sequences, 151,936 ids: one row each 39.4 us, two 36.3, three 36.5, four 38.1, nine 39.1; 170 of 10 with texts of 8000: 55.8, 44.5, 43.3, 42.6, 43.9;
    // 17 of one: 9.2, 8.8)
    const long long all = (long long)slices * a.total_rows, fit = std::min({3ll, (long long)a.total_rows / a.n_seqs, all / 600});
    const int rows_each = (int)std::max({1ll, fit, all / 0x7fffff});    // (a launch takes 2^24 workgroups)
    const long long blocks = (long long)slices * ((a.total_rows + rows_each - 1) / rows_each);
    hipLaunchKernelGGL((logits_adjust_kernel<T, SLICE, VEC, WAY>), dim3((unsigned)blocks), dim3(LOGIT_THREADS), 0, st, a, x, (const T *)logits, out, slices,
                       rows_each);
    VF_LAUNCH_CHECK("logits_adjust");
    return VF_OK;
}

// Results of 100 MB and more go past the caches, which do not hold them until they are read: 200 rows of 151,936 ids and a kernel that reads
// them behind it 99 us for 107; 150 rows (91 MB) would be written faster too (40.6 for 44.9), but read
// slower by more (together 87 for 82).
template <typename T, int SLICE, bool VEC>
int launch(const vf_logits_args &a, const LogitsArrays &x, const void *logits, float *out, hipStream_t st) {
    if constexpr (std::is_same<T, float>::value)
        if (logits == out) return launch_slices<T, SLICE, VEC, IN_PLACE>(a, x, logits, out, st);
    return 4ll * a.total_rows * a.vocab >= 100'000'000 ? launch_slices<T, SLICE, VEC, PAST>(a, x, logits, out, st)
                                                       : launch_slices<T, SLICE, VEC, CACHED>(a, x, logits, out, st);
}

// Ids a workgroup: the text is read once for each slice of a row, so larger slices read it less often and leave fewer workgroups.
template <typename T, bool VEC> int launch(const vf_logits_args &a, const LogitsArrays &x, const void *logits, float *out, hipStream_t st) {
    const long long thousands = (a.vocab + 1023ll) / 1024 * a.total_rows;
    // few of them: one row of 151,936 ids 4.1 us for 4.5, four of 100,003 5.8 for 6.7; eight of 151,936 7.4 for 6.6
    if (thousands <= 800) return launch<T, 1024, VEC>(a, x, logits, out, st);
    // many rows of a sequence each with room for long texts, whose lengths only the device knows (200 rows, texts of 8000: 57.7 us for 63.5, of 2000 46.8
    // for 47.5, of 200 in a history as wide 45.8 for 41.3)
    if (VEC && thousands > 16384 && a.max_history >= 1024 && a.total_rows < 2ll * a.n_seqs) return launch<T, VEC ? 4096 : 2048, VEC>(a, x, logits, out, st);
    return launch<T, 2048, VEC>(a, x, logits, out, st);
}

template <typename T> int launch(const vf_logits_args &a, const LogitsArrays &x, const void *logits, float *out, hipStream_t st) {
    // four ids at a time need rows that start at a multiple of four elements
    const bool vec = !(a.vocab & 3) && !((a.in_stride | a.out_stride) & 3) && !((uintptr_t)logits & (4 * sizeof(T) - 1)) && !((uintptr_t)out & 15);
    return vec ? launch<T, true>(a, x, logits, out, st) : launch<T, false>(a, x, logits, out, st);
}

// Whether a row of `a` (bytes a_row, a_step apart) shares bytes with a row of `b`, both of `rows` rows: rows of one may lie between those of the other.
bool rows_overlap(uintptr_t a, int64_t a_row, int64_t a_step, uintptr_t b, int64_t b_row, int64_t b_step, int rows) {
    if (a >= b + (rows - 1) * b_step + b_row || b >= a + (rows - 1) * a_step + a_row) return false;
    for (int r = 0; r < rows; ++r) {
        // of the rows of b that end behind the start of this one, the first
        const int64_t start = (int64_t)(a - b) + r * a_step, first = start < b_row ? 0 : (start - b_row) / b_step + 1;
        if (first < rows && first * b_step < start + a_row) return true;
    }
    return false;
}

}  // namespace

extern "C" int vf_logits_adjust(const vf_logits_args *args, const void *logits_dev, const int32_t *row_off_dev, float *out_dev,
                                const float *penalties_dev, const int32_t *history_dev, const int32_t *history_len_dev,
                                const int32_t *prompt_len_dev, const int32_t *tokens_dev, const int32_t *bias_off_dev,
                                const int32_t *bias_id_dev, const float *bias_dev, const uint32_t *mask_dev,
                                const int32_t *mask_row_dev, void *stream) {
    if (!args) return vf_fail(VF_ERR_ARG, "vf_logits_adjust: NULL argument");
    const vf_logits_args &a = *args;
    if (a.dtype != VF_F32 && a.dtype != VF_BF16) return vf_fail(VF_ERR_ARG, "vf_logits_adjust: dtype %d", a.dtype);
    if (a.n_seqs < 1 || a.n_seqs > VF_PACKED_MAX_SEQS || a.total_rows < 0 || a.total_rows > VF_PACKED_MAX_ROWS)
        return vf_fail(VF_ERR_ARG, "vf_logits_adjust: %d sequences, %d rows", a.n_seqs, a.total_rows);
    if (a.vocab < 1 || a.vocab > VF_LOGITS_MAX_VOCAB || a.in_stride < a.vocab || a.out_stride < a.vocab)
        return vf_fail(VF_ERR_ARG, "vf_logits_adjust: vocabulary %d, strides %lld, %lld", a.vocab, (long long)a.in_stride, (long long)a.out_stride);
    if (a.total_rows == 0) return VF_OK;
    if (!logits_dev || !row_off_dev || !out_dev) return vf_fail(VF_ERR_ARG, "vf_logits_adjust: NULL argument");
    if ((void *)out_dev == logits_dev && (a.dtype != VF_F32 || a.in_stride != a.out_stride))
        return vf_fail(VF_ERR_ARG, "vf_logits_adjust: in place with another type or stride");
    if (history_dev && (!history_len_dev || a.max_history < 0 || a.max_history > VF_LOGITS_MAX_HISTORY || a.history_stride < a.max_history))
        return vf_fail(VF_ERR_ARG, "vf_logits_adjust: history of at most %d tokens, stride %lld, lengths %p", a.max_history, (long long)a.history_stride,
                       (const void *)history_len_dev);
    if (!history_dev && prompt_len_dev) return vf_fail(VF_ERR_ARG, "vf_logits_adjust: prompt lengths without a history");
    if ((history_dev || tokens_dev) && !penalties_dev) history_dev = tokens_dev = nullptr;    // nothing counts them
    if (bias_off_dev && (a.bias_entries < 0 || a.bias_entries > VF_LOGITS_MAX_BIASES || (a.bias_entries > 0 && (!bias_id_dev || !bias_dev))))
        return vf_fail(VF_ERR_ARG, "vf_logits_adjust: %d biases", a.bias_entries);
    if (((uintptr_t)logits_dev & (a.dtype == VF_F32 ? 3 : 1)) | ((uintptr_t)out_dev & 3))
        return vf_fail(VF_ERR_UNSUPPORTED, "vf_logits_adjust: addresses are multiples of an element");
    const int es = a.dtype == VF_F32 ? 4 : 2;
    if ((const void *)out_dev != logits_dev && rows_overlap((uintptr_t)logits_dev, (int64_t)a.vocab * es, a.in_stride * es, (uintptr_t)out_dev,
                                                            (int64_t)a.vocab * 4, a.out_stride * 4, a.total_rows))
        return vf_fail(VF_ERR_ARG, "vf_logits_adjust: out shares memory with the logits and is not them");
    if (mask_dev && (a.mask_rows < 0 || a.mask_stride < (a.vocab + 31) / 32 || (!mask_row_dev && a.mask_rows < a.total_rows)))
        return vf_fail(VF_ERR_ARG, "vf_logits_adjust: %d masks, stride %lld", a.mask_rows, (long long)a.mask_stride);
    const LogitsArrays x = {row_off_dev, penalties_dev, history_dev, history_len_dev, prompt_len_dev, tokens_dev, bias_off_dev, bias_id_dev, bias_dev,
                            mask_dev, mask_row_dev};
    return a.dtype == VF_F32 ? launch<float>(a, x, logits_dev, out_dev, (hipStream_t)stream)
                             : launch<bf16_t>(a, x, logits_dev, out_dev, (hipStream_t)stream);
}
