// Penalties for repeated tokens, biases and grammar masks on the logits of packed rows.
#include <algorithm>

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

template <typename T> struct alignas(4 * sizeof(T)) Four { T v[4]; };

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

struct Penalty { float repetition, presence, frequency; };

// (count: bit 0: seen in the prompt; above: how often given)
__device__ __forceinline__ float adjusted(float z, unsigned count, float bias, bool allowed, const Penalty &p) {
    if (count) z = z > 0.f ? z / p.repetition : z * p.repetition;
    if (count >> 1) z -= p.presence + p.frequency * (float)(count >> 1);
    z += bias;
    return allowed ? z : -INFINITY;
}

// A workgroup has SLICE ids of some rows.  Two tables in LDS hold how often the sequence's text has each id and its bias; they are made
// once for the rows of a sequence, and a row adds its own token.  Counts are whole numbers, so the order of the additions does not
// matter, and of several biases of an id the last of the list is found as a maximum over their places.
template <typename T, int SLICE, bool VEC>
__global__ __launch_bounds__(LOGIT_THREADS) void logits_adjust_kernel(vf_logits_args a, LogitsArrays x, const T *logits, float *out, int slices,
                                                                      int rows_each) {
    constexpr int EACH = SLICE / LOGIT_THREADS;
    __shared__ __align__(16) unsigned count[SLICE];
    __shared__ __align__(16) float bias[SLICE];
    const int tid = threadIdx.x, chunk = blockIdx.x / slices, v0 = (blockIdx.x - chunk * slices) * SLICE;
    const int r0 = chunk * rows_each, r1 = (int)min((long long)r0 + rows_each, (long long)a.total_rows);
    // ids of a thread: EACH / 4 times four in a row, or EACH of them LOGIT_THREADS apart
    auto id_of = [&](int i) { return VEC ? i / 4 * 4 * LOGIT_THREADS + tid * 4 + i % 4 : i * LOGIT_THREADS + tid; };
    int seq = -1, end = 0;     // the tables' sequence, the end of its rows
    bool counted = false, biased = false, inside = false;
    Penalty p{1.f, 0.f, 0.f};
    for (int r = r0; r < r1; ++r) {
        T z[EACH];
        const T *zr = logits + (size_t)r * a.in_stride + v0;
#pragma unroll
        for (int i = 0; i < EACH; i += VEC ? 4 : 1) {
            if constexpr (VEC) {
                if (v0 + id_of(i) < a.vocab) *reinterpret_cast<Four<T> *>(z + i) = *reinterpret_cast<const Four<T> *>(zr + id_of(i));
            } else {
                if (v0 + id_of(i) < a.vocab) z[i] = zr[id_of(i)];
            }
        }
        if (r >= end) {        // the first row, or the first of another sequence
            seq = sequence_of(x.row_off, a.n_seqs, r);
            inside = seq >= 0 && seq < a.n_seqs;
            const int first = inside ? x.row_off[seq] : 0;
            end = inside ? x.row_off[seq + 1] : (seq < 0 ? x.row_off[0] : a.total_rows);
            inside = inside && first >= 0 && end > r;
            if (end <= r) end = r + 1;
            if (!inside) continue;
            if (x.penalties) p = Penalty{x.penalties[3 * seq], x.penalties[3 * seq + 1], x.penalties[3 * seq + 2]};
            counted = x.penalties && (p.repetition != 1.f || p.presence != 0.f || p.frequency != 0.f);
            const int b0 = x.bias_off ? max(x.bias_off[seq], 0) : 0, b1 = x.bias_off ? min(x.bias_off[seq + 1], a.bias_entries) : 0;
            biased = b0 < b1;
            __syncthreads();
            if (counted || biased) {
                for (int i = tid; i < SLICE; i += LOGIT_THREADS) {
                    count[i] = 0;
                    bias[i] = 0.f;
                }
                __syncthreads();
            }
            if (biased) {
                for (int i = b0 + tid; i < b1; i += LOGIT_THREADS) {
                    const unsigned d = (unsigned)x.bias_id[i] - v0;
                    if (d < SLICE) atomicMax(&count[d], (unsigned)(i - b0) + 1);
                }
                __syncthreads();
                for (int i = b0 + tid; i < b1; i += LOGIT_THREADS) {
                    const unsigned d = (unsigned)x.bias_id[i] - v0;
                    if (d < SLICE && count[d] == (unsigned)(i - b0) + 1) bias[d] = x.bias[i];
                }
                __syncthreads();
                if (counted) {
                    for (int i = tid; i < SLICE; i += LOGIT_THREADS) count[i] = 0;
                    __syncthreads();
                }
            }
            if (counted) {
                if (x.history) {
                    const int n = min(max(x.history_len[seq], 0), a.max_history), prompt = x.prompt_len ? min(max(x.prompt_len[seq], 0), n) : 0;
                    const int32_t *text = x.history + (size_t)seq * a.history_stride;
                    for (int i0 = tid; i0 < n; i0 += 8 * LOGIT_THREADS) {
                        int id[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) id[j] = text[min(i0 + j * LOGIT_THREADS, n - 1)];
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const unsigned d = (unsigned)id[j] - v0;
                            const int i = i0 + j * LOGIT_THREADS;
                            if (d < SLICE && i < n) {
                                if (i < prompt) atomicOr(&count[d], 1u);
                                else atomicAdd(&count[d], 2u);
                            }
                        }
                    }
                }
                if (x.tokens)
                    for (int i = first + tid; i < r; i += LOGIT_THREADS) {
                        const unsigned d = (unsigned)x.tokens[i] - v0;
                        if (d < SLICE) atomicAdd(&count[d], 2u);
                    }
                __syncthreads();
            }
        }
        if (!inside) continue;
        if (counted && x.tokens) {
            const unsigned d = (unsigned)x.tokens[r] - v0;
            if (d < SLICE) {
                __syncthreads();     // the rows before have been read
                if (tid == 0) count[d] += 2;
                __syncthreads();
            }
        }
        const int m = x.mask ? (x.mask_row ? x.mask_row[r] : r) : -1;
        const bool masked = m >= 0 && m < a.mask_rows;
        const uint32_t *bits = x.mask + (masked ? (size_t)m * a.mask_stride + v0 / 32 : 0);
        float *to = out + (size_t)r * a.out_stride + v0;
#pragma unroll
        for (int i = 0; i < EACH; i += VEC ? 4 : 1) {
            if (v0 + id_of(i) >= a.vocab) continue;
            const uint32_t word = masked ? bits[id_of(i) / 32] >> id_of(i) % 32 : 0xffffffffu;
            if constexpr (VEC) {
                const Four<unsigned> c = counted ? *reinterpret_cast<const Four<unsigned> *>(count + id_of(i)) : Four<unsigned>{};
                const Four<float> b = biased ? *reinterpret_cast<const Four<float> *>(bias + id_of(i)) : Four<float>{};
                Four<float> y;
#pragma unroll
                for (int j = 0; j < 4; ++j) y.v[j] = adjusted(to_f32(z[i + j]), c.v[j], b.v[j], word >> j & 1, p);
                *reinterpret_cast<Four<float> *>(to + id_of(i)) = y;
            } else {
                to[id_of(i)] = adjusted(to_f32(z[i]), counted ? count[id_of(i)] : 0u, biased ? bias[id_of(i)] : 0.f, word & 1, p);
            }
        }
    }
}

template <typename T, int SLICE, bool VEC>
int launch(const vf_logits_args &a, const LogitsArrays &x, const void *logits, float *out, hipStream_t st) {
    const int slices = (a.vocab + SLICE - 1) / SLICE;
    const long long all = (long long)slices * a.total_rows;
    const int rows_each = (int)std::max(1ll, std::min((long long)a.total_rows, all / 4096));
    const long long blocks = (long long)slices * ((a.total_rows + rows_each - 1) / rows_each);
    hipLaunchKernelGGL((logits_adjust_kernel<T, SLICE, VEC>), dim3((unsigned)blocks), dim3(LOGIT_THREADS), 0, st, a, x, (const T *)logits, out, slices,
                       rows_each);
    VF_LAUNCH_CHECK("logits_adjust");
    return VF_OK;
}

template <typename T> int launch(const vf_logits_args &a, const LogitsArrays &x, const void *logits, float *out, hipStream_t st) {
    // four ids at a time need rows that start at a multiple of four elements
    const bool vec = !(a.vocab & 3) && !((a.in_stride | a.out_stride) & 3) && !((uintptr_t)logits & (4 * sizeof(T) - 1)) && !((uintptr_t)out & 15);
    return vec ? launch<T, 2048, true>(a, x, logits, out, st) : launch<T, 2048, false>(a, x, logits, out, st);
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
    if (bias_off_dev && (a.bias_entries < 0 || (a.bias_entries > 0 && (!bias_id_dev || !bias_dev))))
        return vf_fail(VF_ERR_ARG, "vf_logits_adjust: %d biases", a.bias_entries);
    if (mask_dev && (a.mask_rows < 0 || a.mask_stride < (a.vocab + 31) / 32 || (!mask_row_dev && a.mask_rows < a.total_rows)))
        return vf_fail(VF_ERR_ARG, "vf_logits_adjust: %d masks, stride %lld", a.mask_rows, (long long)a.mask_stride);
    if (((uintptr_t)logits_dev & (a.dtype == VF_F32 ? 3 : 1)) | ((uintptr_t)out_dev & 3))
        return vf_fail(VF_ERR_UNSUPPORTED, "vf_logits_adjust: addresses are multiples of an element");
    const LogitsArrays x = {row_off_dev, penalties_dev, history_dev, history_len_dev, prompt_len_dev, tokens_dev, bias_off_dev, bias_id_dev, bias_dev,
                            mask_dev, mask_row_dev};
    return a.dtype == VF_F32 ? launch<float>(a, x, logits_dev, out_dev, (hipStream_t)stream)
                             : launch<bf16_t>(a, x, logits_dev, out_dev, (hipStream_t)stream);
}
