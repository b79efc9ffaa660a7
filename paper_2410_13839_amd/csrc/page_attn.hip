// Attention of new tokens over a paged cache (mtp_pages_attention): causal
// chunks of any length (one token to whole prompts), or full attention over
// another sequence's states.  See include/mtp.h for the operator's definition.
//
//   out[t][h] = sum_j p_j V[j] / sum_j p_j,  p_j = exp2(s_j - m),
//   s_j = scale log2(e) q . K[j],  m the running maximum
//
// in one pass over the keys.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/mtp.h"
#include "common.h"
#include "wave.h"

namespace mtp {

int cache_check(const mtp_cache& c);

namespace {

constexpr int PG = 16;
constexpr float LOG2E = 1.4426950408889634f;

// The row whose tokens include t, or -1: the last c with row_start[c] <= t,
// found by the whole wave (64 candidates a round).
__device__ __forceinline__ int row_of_token(const mtp_attention_args& a, int t) {
    int lo = 0, n = a.n_rows;                    // the answer lies in [lo, lo + n)
    const int lane = threadIdx.x & 63;
    while (n > 1) {
        const int step = (n + 63) / 64;
        const int i = lane * step;
        const bool le = i < n && a.row_start[lo + i] <= t;
        const int k = __popcll(__ballot(le));
        if (k == 0) return -1;
        lo += (k - 1) * step;
        n = min(step, n - (k - 1) * step);
    }
    return t >= a.row_start[lo] && t < a.row_start[lo + 1] ? lo : -1;
}

// One wave per (token, head).
template <typename T, int D>
__global__ __launch_bounds__(64) void attn_simple_kernel(mtp_attention_args a) {
    const int t = blockIdx.x, head = blockIdx.y, lane = threadIdx.x;
    const int c = row_of_token(a, t);
    if (c < 0) return;
    const int s0 = max(a.row_start[c], 0), s1 = min(a.row_start[c + 1], a.n_tokens);
    const int kv = max(0, min(a.kv_len[c], PG * a.max_pages));
    const int pos = kv - (s1 - s0) + (t - s0);
    int hi = kv, lo = 0;
    if (a.mode == MTP_ATTN_CAUSAL) {
        hi = min(kv, pos + 1);
        if (a.window > 0) lo = max(0, pos - a.window + 1);
    }
    const int H = a.cache.n_kv_heads, hk = head / (a.n_heads / H);
    const T* q = (const T*)a.q + (int64_t)t * a.q_stride + head * D;
    const T* pool = (const T*)a.cache.pool;
    float m = -INFINITY, l = 0.f, acc[D / 64] = {};
    for (int j = lo; j < hi; ++j) {
        const int pg = a.table[(size_t)c * a.max_pages + j / PG];
        if (pg < 0 || pg >= a.cache.num_pages) continue;
        const T* K = pool + ((size_t)pg * 2 * H + hk) * PG * D + (j % PG) * D;
        const T* V = pool + ((size_t)pg * 2 * H + H + hk) * PG * D;
        float s = 0.f;
        for (int d = lane; d < D; d += 64) s += ActIO<T>::load(q + d) * ActIO<T>::load(K + d);
        s = wave_sum64(s) * (a.scale * LOG2E);
        const float mn = fmaxf(m, s);
        const float r = m == -INFINITY ? 0.f : exp2f(m - mn), p = exp2f(s - mn);
        m = mn;
        l = l * r + p;
        for (int i = 0; i < D / 64; ++i) {
            const int d = lane + 64 * i;
            acc[i] = acc[i] * r + p * ActIO<T>::load(V + (sizeof(T) == 2 ? d * PG + j % PG : (j % PG) * D + d));
        }
    }
    T* o = (T*)a.out + (int64_t)t * a.out_stride + head * D;
    const float inv = l > 0.f ? 1.f / l : (m == -INFINITY ? 0.f : NAN);
    for (int i = 0; i < D / 64; ++i) ActIO<T>::store(o + lane + 64 * i, acc[i] * inv);
}

bool aligned(const void* p, uintptr_t n) { return p && ((uintptr_t)p & (n - 1)) == 0; }

int attn_check(const mtp_attention_args* a) {
    if (!a) return MTP_EINVAL;
    const int rc = cache_check(a->cache);
    if (rc != MTP_OK) return rc;
    if (a->n_rows < 0 || a->n_rows > 4096 || a->max_pages < 1 || a->max_pages > 65536 || a->n_tokens < 0 ||
        a->n_tokens >= (1 << 24) || a->n_heads < 1 || a->n_heads > 1024 || a->n_heads % a->cache.n_kv_heads)
        return MTP_EINVAL;
    if (a->mode != MTP_ATTN_CAUSAL && a->mode != MTP_ATTN_FULL) return MTP_EINVAL;
    if (a->window < 0 || (a->mode == MTP_ATTN_FULL && a->window != 0) || a->max_kv < 0 || !isfinite(a->scale)) return MTP_EINVAL;
    return MTP_OK;
}

}  // namespace
}  // namespace mtp

extern "C" {

int mtp_pages_attention_workspace_size(const mtp_attention_args* args, uint64_t* bytes) {
    const int rc = mtp::attn_check(args);
    if (rc != MTP_OK || !bytes) return MTP_EINVAL;
    *bytes = 0;
    return MTP_OK;
}

int mtp_pages_attention(const mtp_attention_args* args, void* hip_stream) {
    using namespace mtp;
    const int rc = attn_check(args);
    if (rc != MTP_OK) return rc;
    const mtp_attention_args& a = *args;
    if (a.n_rows == 0 || a.n_tokens == 0) return MTP_OK;
    const int64_t per = a.cache.dtype == MTP_DTYPE_BF16 ? 8 : 4, row = (int64_t)a.n_heads * a.cache.head_dim;
    if (!aligned(a.table, 4) || !aligned(a.row_start, 4) || !aligned(a.kv_len, 4) || !aligned(a.q, 16) ||
        !aligned(a.out, 16) || a.q_stride < row || a.out_stride < row || a.q_stride % per || a.out_stride % per)
        return MTP_EINVAL;
    const dim3 grid(a.n_tokens, a.n_heads), block(64);
    hipStream_t st = (hipStream_t)hip_stream;
    if (a.cache.dtype == MTP_DTYPE_BF16) {
        if (a.cache.head_dim == 64) hipLaunchKernelGGL((attn_simple_kernel<bf16_t, 64>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((attn_simple_kernel<bf16_t, 128>), grid, block, 0, st, a);
    } else {
        if (a.cache.head_dim == 64) hipLaunchKernelGGL((attn_simple_kernel<float, 64>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((attn_simple_kernel<float, 128>), grid, block, 0, st, a);
    }
    return hipGetLastError() == hipSuccess ? MTP_OK : MTP_EHIP;
}

}  // extern "C"
