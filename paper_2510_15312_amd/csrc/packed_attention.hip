// Causal attention of packed rows with grouped heads over the page pool: whole prompts, chunks behind a cached prefix,
// drafts and single tokens of many sequences in one call.
#include <algorithm>
#include <cmath>

#include "vf_internal.h"

namespace {

struct PackedAttn {
    vf_packed_args a;
    const void *q, *kv;
    const int32_t *table, *row_off, *kv_len;
    void *out;
};

// One wavefront per row and query head: a key per lane for the scores, HD / 64 elements per lane for the sums.
template <typename T, int HD>
__global__ __launch_bounds__(64) void attention_plain_kernel(PackedAttn p) {
    const vf_packed_args &a = p.a;
    __shared__ float qs[HD];
    const int row = blockIdx.x, head = blockIdx.y, lane = threadIdx.x, kvh = head / (a.n_q_heads / a.n_kv_heads);
    int b = 0;
    while (b < a.n_seqs && row >= p.row_off[b + 1]) ++b;
    if (b == a.n_seqs || row < p.row_off[b]) return;
    const int rows = min(p.row_off[b + 1], a.total_rows) - p.row_off[b];
    const int last = min(p.kv_len[b] - rows + row - p.row_off[b], min(p.kv_len[b], a.max_pages * VF_TILE) - 1);
    const T *q = (const T *)p.q + row * a.q_stride + head * HD, *kv = (const T *)p.kv;
    for (int d = lane; d < HD; d += 64) qs[d] = to_f32(q[d]);
    __syncthreads();
    float m = -INFINITY, l = 0.f, acc[HD / 64] = {};
    for (int t0 = 0; t0 <= last; t0 += VF_TILE) {
        const int page = p.table[(size_t)b * a.table_stride + t0 / VF_TILE];
        if (page < 0 || page >= a.pool_pages) continue;
        float s = -INFINITY;
        if (t0 + lane <= last) {
            s = 0.f;
            for (int d = 0; d < HD; ++d) s += qs[d] * to_f32(kv[kv_k_index(0, 0, page, a.n_kv_heads, kvh, lane, d, HD)]);
            s *= a.scale;
        }
        float mx = s;
        for (int d = 32; d; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d, 64));
        const float m_new = fmaxf(m, mx), keep = m == -INFINITY ? 0.f : expf(m - m_new);
        float w = t0 + lane <= last ? expf(s - m_new) : 0.f;
        l = l * keep + w;
        for (int i = 0; i < HD / 64; ++i) acc[i] *= keep;
        m = m_new;
        for (int j = 0; j <= min(VF_TILE - 1, last - t0); ++j) {
            const float wj = __shfl(w, j, 64);
            for (int i = 0; i < HD / 64; ++i)
                acc[i] += wj * to_f32(kv[kv_v_index(0, 0, page, a.n_kv_heads, kvh, j, lane + 64 * i, HD)]);
        }
    }
    for (int d = 32; d; d >>= 1) l += __shfl_xor(l, d, 64);
    for (int i = 0; i < HD / 64; ++i)
        ((T *)p.out)[row * a.out_stride + head * HD + lane + 64 * i] = from_f32<T>(m == -INFINITY ? 0.f : acc[i] / l);
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
    if (!std::isfinite(a.scale)) return vf_fail(VF_ERR_ARG, "%s: scale %g", name, a.scale);
    const int64_t w = (int64_t)a.n_q_heads * a.head_dim;
    if (a.q_stride < w || a.out_stride < w)
        return vf_fail(VF_ERR_ARG, "%s: rows overlap (strides %lld, %lld)", name, (long long)a.q_stride, (long long)a.out_stride);
    if ((a.q_stride | a.out_stride) * (a.dtype == VF_BF16 ? 2 : 4) & 15)
        return vf_fail(VF_ERR_UNSUPPORTED, "%s: strides are multiples of 16 bytes", name);
    return VF_OK;
}

}  // namespace

extern "C" {

size_t vf_attention_packed_workspace(const vf_packed_args *args) {
    if (check("vf_attention_packed_workspace", args) != VF_OK) return (size_t)-1;
    return 0;
}

int vf_attention_packed(const vf_packed_args *args, const void *q_dev, const void *kv_layer_dev, const int32_t *block_table_dev,
                        const int32_t *row_off_dev, const int32_t *kv_len_dev, void *out_dev, void *workspace_dev, size_t workspace_bytes,
                        void *stream) {
    if (int rc = check("vf_attention_packed", args)) return rc;
    PackedAttn p = {*args, q_dev, kv_layer_dev, block_table_dev, row_off_dev, kv_len_dev, out_dev};
    if (p.a.total_rows == 0) return VF_OK;
    if (!q_dev || !kv_layer_dev || !block_table_dev || !row_off_dev || !kv_len_dev || !out_dev)
        return vf_fail(VF_ERR_ARG, "vf_attention_packed: NULL argument");
    if (((uintptr_t)q_dev | (uintptr_t)kv_layer_dev | (uintptr_t)out_dev) & 15)
        return vf_fail(VF_ERR_UNSUPPORTED, "vf_attention_packed: addresses are multiples of 16 bytes");
    if (p.a.scale == 0.f) p.a.scale = 1.0f / sqrtf((float)p.a.head_dim);
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid(p.a.total_rows, p.a.n_q_heads);
    const auto kernel = p.a.dtype == VF_BF16 ? (p.a.head_dim == 128 ? attention_plain_kernel<bf16_t, 128> : attention_plain_kernel<bf16_t, 64>)
                                             : (p.a.head_dim == 128 ? attention_plain_kernel<float, 128> : attention_plain_kernel<float, 64>);
    hipLaunchKernelGGL(kernel, grid, dim3(64), 0, st, p);
    VF_LAUNCH_CHECK("attention_packed");
    return VF_OK;
}

}  // extern "C"
