// Beam search's selection (mtp_beam_select).
//
//   lp[v] = x[v] - (M + log sum_v exp(x[v] - M)),  M = max x
//
// A beam's best candidates are its largest logits whatever its normaliser, so
// one pass per beam row finds both; a second step per request ranks the beams'
// candidates against each other in float64.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/mtp.h"
#include "common.h"
#include "wave.h"

namespace mtp {
namespace {

constexpr int BT = 256;                  // threads per beam row
constexpr int MAX_BEAMS = 32;

struct BeamWs {
    double* lse;                         // [rows]
    float* val;                          // [rows][beams] a row's best logits, best first
    int32_t* idx;                        // [rows][beams]
};

uint64_t beam_carve(const mtp_beam_args& a, BeamWs* w) {
    const uint64_t rows = (uint64_t)a.n_requests * a.beams;
    uint64_t o = 0;
    auto take = [&](uint64_t bytes) { uint64_t r = o; o = (o + bytes + 255) & ~uint64_t(255); return r; };
    const uint64_t l = take(rows * 8), v = take(rows * a.beams * 4), i = take(rows * a.beams * 4);
    if (w) {
        char* p = (char*)a.workspace;
        w->lse = (double*)(p + l); w->val = (float*)(p + v); w->idx = (int32_t*)(p + i);
    }
    return o;
}

// The logit as the selection sees it.
__device__ __forceinline__ float beam_logit(const mtp_beam_args& a, const float* x, int v, bool mask_eos) {
    const float f = x[v];
    return (f != f || (mask_eos && v == a.eos_id)) ? -INFINITY : f;
}

// Best first: larger value, then lower index.
__device__ __forceinline__ bool before(float va, int ia, float vb, int ib) { return va > vb || (va == vb && ia < ib); }

__global__ __launch_bounds__(BT) void beam_row_kernel(mtp_beam_args a, BeamWs w) {
    __shared__ float s_v[BT / 64];
    __shared__ int s_i[BT / 64];
    __shared__ double s_s[BT / 64];
    const int row = blockIdx.x, tid = threadIdx.x;
    if (a.done[row] > 0) return;
    const float* x = a.logits + (int64_t)row * a.ld;
    const bool mask = a.len[row] < a.eos_min;
    float pv = INFINITY;                 // the last one taken
    int pi = -1;
    const int n = min(a.beams, a.vocab);
    for (int k = 0; k < n; ++k) {
        float bv = -INFINITY;
        int bi = 0x7fffffff;
        for (int v = tid; v < a.vocab; v += BT) {
            const float f = beam_logit(a, x, v, mask);
            if (before(pv, pi, f, v) && before(f, v, bv, bi)) { bv = f; bi = v; }
        }
        wave_argmax(bv, bi);
        if ((tid & 63) == 0) { s_v[tid >> 6] = bv; s_i[tid >> 6] = bi; }
        __syncthreads();
        for (int i = 0; i < BT / 64; ++i)
            if (i == 0 || before(s_v[i], s_i[i], bv, bi)) { bv = s_v[i]; bi = s_i[i]; }
        __syncthreads();
        if (tid == 0) { w.val[(size_t)row * a.beams + k] = bv; w.idx[(size_t)row * a.beams + k] = bi; }
        pv = bv; pi = bi;
        if (k == 0) {
            double s = 0.0;
            for (int v = tid; v < a.vocab; v += BT) s += (double)expf(beam_logit(a, x, v, mask) - bv);
            for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
            if ((tid & 63) == 0) s_s[tid >> 6] = s;
            __syncthreads();
            if (tid == 0) {
                s = 0.0;
                for (int i = 0; i < BT / 64; ++i) s += s_s[i];
                w.lse[row] = (double)bv + log(s);
            }
        }
    }
}

__global__ __launch_bounds__(64) void beam_merge_kernel(mtp_beam_args a, BeamWs w) {
    __shared__ double s_den[MAX_BEAMS], s_lse[MAX_BEAMS];
    __shared__ float s_score[MAX_BEAMS];
    __shared__ int s_len[MAX_BEAMS], s_done[MAX_BEAMS];
    const int r = blockIdx.x, lane = threadIdx.x, W = a.beams, n = min(W, a.vocab);
    if (lane < W) {
        const int row = r * W + lane;
        const int dn = a.done[row] > 0;
        const int len = a.len[row] + (dn ? 0 : 1);
        s_done[lane] = dn; s_len[lane] = len; s_score[lane] = a.score[row];
        s_lse[lane] = dn ? 0.0 : w.lse[row];
        s_den[lane] = pow((double)max(len, 1), (double)a.alpha);
    }
    __syncthreads();
    double pr = INFINITY;
    int64_t pf = -1;
    for (int k = 0; k < W; ++k) {
        double br = -INFINITY, bt = -INFINITY;
        int64_t bf = INT64_MAX;
        for (int i = lane; i < W * n; i += 64) {
            const int b = i / n, j = i % n;
            int tok;
            double total;
            if (s_done[b]) {
                // itself first, then the tokens it cannot take
                tok = j == 0 ? a.eos_id : (j - 1 < a.eos_id ? j - 1 : j);
                total = j == 0 ? (double)s_score[b] : -INFINITY;
            } else {
                const size_t at = ((size_t)r * W + b) * W + j;
                tok = w.idx[at];
                total = (double)s_score[b] + ((double)w.val[at] - s_lse[b]);
            }
            if (!(total < INFINITY)) total = -INFINITY;      // NaN too
            double rank = total / s_den[b];
            if (!(rank == rank)) rank = -INFINITY;       // -infinity by an overflowed length term
            const int64_t flat = (int64_t)b * a.vocab + tok;
            const bool later = rank < pr || (rank == pr && flat > pf);
            if (later && (rank > br || (rank == br && flat < bf))) { br = rank; bt = total; bf = flat; }
        }
        for (int o = 32; o; o >>= 1) {
            const double orr = __shfl_xor(br, o), ot = __shfl_xor(bt, o);
            const int64_t of = __shfl_xor((long long)bf, o);
            if (orr > br || (orr == br && of < bf)) { br = orr; bt = ot; bf = of; }
        }
        pr = br; pf = bf;
        if (lane == 0) {
            const int b = (int)(bf / a.vocab), tok = (int)(bf % a.vocab), o = r * W + k;
            a.out_score[o] = (float)bt;
            a.out_len[o] = s_len[b];
            a.out_done[o] = s_done[b] | (tok == a.eos_id ? 1 : 0);
            a.out_parent[o] = r * W + b;
            a.out_token[o] = tok;
        }
    }
}

bool aligned(const void* p, uintptr_t n) { return p && ((uintptr_t)p & (n - 1)) == 0; }

int beam_check(const mtp_beam_args* a) {
    if (!a) return MTP_EINVAL;
    if (a->beams < 1 || a->beams > MAX_BEAMS || a->n_requests < 0 || (int64_t)a->n_requests * a->beams > 65536 ||
        a->vocab < 1 || a->vocab >= (1 << 24) || a->eos_id < 0 || a->eos_id >= a->vocab || !(a->alpha >= 0.f) ||
        !isfinite(a->alpha))
        return MTP_EINVAL;
    return MTP_OK;
}

}  // namespace
}  // namespace mtp

extern "C" {

int mtp_beam_select_workspace_size(const mtp_beam_args* args, uint64_t* bytes) {
    const int rc = mtp::beam_check(args);
    if (rc != MTP_OK || !bytes) return MTP_EINVAL;
    *bytes = mtp::beam_carve(*args, nullptr);
    return MTP_OK;
}

int mtp_beam_select(const mtp_beam_args* args, void* hip_stream) {
    using namespace mtp;
    const int rc = beam_check(args);
    if (rc != MTP_OK) return rc;
    const mtp_beam_args& a = *args;
    if (a.n_requests == 0) return MTP_OK;
    if (!aligned(a.logits, 4) || !aligned(a.score, 4) || !aligned(a.len, 4) || !aligned(a.done, 4) ||
        !aligned(a.out_score, 4) || !aligned(a.out_len, 4) || !aligned(a.out_done, 4) || !aligned(a.out_parent, 4) ||
        !aligned(a.out_token, 4) || !aligned(a.workspace, 256) || a.ld < a.vocab)
        return MTP_EINVAL;
    BeamWs w{};
    if (beam_carve(a, &w) > a.workspace_bytes) return MTP_ENOMEM;
    hipStream_t st = (hipStream_t)hip_stream;
    hipLaunchKernelGGL(beam_row_kernel, dim3(a.n_requests * a.beams), dim3(BT), 0, st, a, w);
    hipLaunchKernelGGL(beam_merge_kernel, dim3(a.n_requests), dim3(64), 0, st, a, w);
    return hipGetLastError() == hipSuccess ? MTP_OK : MTP_EHIP;
}

}  // extern "C"
