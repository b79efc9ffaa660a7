// Beam search's selection (mtp_beam_select).
//
//   lp[v] = x[v] - (M + log sum_v exp(x[v] - M)),  M = max x
//
// A beam's best candidates are its largest logits whatever its normaliser, so
// one pass over the logits finds both.  One wave takes a chunk of 2048 logits
// into registers (32 loads in flight a lane), sums their exponentials and
// keeps the chunk's `beams` best in order: maxima of lanes or groups of them
// bound the last of those from below, what reaches the bound is gathered into LDS
// (a few dozen logits) and taken best first.  A request's workgroup then merges
// the sorted lists of each beam's chunks, and the beams' lists in float64.  With
// few chunks all of it is one launch.
// What bounds it: 16 requests of 8 beams over 65,536 logits (34 MB) take 11.0 us
// for the chunks (3.1 TB/s; 4096 waves load at once and then compute) and 7.7 us
// for the merge, a chain of loads, a float64 exponential, logarithm and power, and
// eight rounds of a wave maximum per beam.  A beam's lists are merged head by
// head, a lane a chunk (1 request of 8 beams over 131,072 logits 15.5 us; 28.8 us
// with all entries compared every round).  One request of
// 4 beams over 1025 logits 8 us: the launch and the same chain.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/mtp.h"
#include "common.h"
#include "launch.h"
#include "wave.h"

namespace mtp {
namespace {

constexpr int MAX_BEAMS = 32;
constexpr int NV = 32;                   // logits per lane
constexpr int CHUNK = 64 * NV;           // logits per wave
constexpr int CAP = 256;                 // gathered candidates per wave
// Up to this many beams a chunk's bound comes from groups of lanes (4 beams over
// 32,000 logits 12.7 us either way; 5 beams 19.0 us with groups and 17.0 us with
// the lanes' maxima, 16 over 50,000 37 and 31 us).
constexpr int FEW_BEAMS = 4;
// Up to this many beams the next ones are found by counting places, a thread per
// candidate and other beam (8 beams over 65,536 logits 20.7 us, 21.5 us head by
// head; 16 over 2000 18.0 and 16.9 us, 32 over 32,000 127 and 56 us).
constexpr int PLACED = 12;
// Chunks per request up to which one launch does everything, a wave each (8
// requests of 4 beams over 16,384 logits, 32 chunks: 18.5 us, 12.9 us in two
// launches; 64 of 8 over 1025, 8 chunks: 10.3 and 11.4 us).
constexpr int FUSED_UNITS = 16;
constexpr float LOG2E = 1.4426950408889634f;

struct BeamWs {
    double* sum;                         // [rows][chunks] sum of exp(x - max)
    float* max;                          // [rows][chunks]
    float2* list;                        // [rows][chunks][beams] (logit, index bits), best first
};

int beam_chunks(int vocab) { return (vocab + CHUNK - 1) / CHUNK; }

uint64_t beam_carve(const mtp_beam_args& a, BeamWs* w) {
    const uint64_t units = (uint64_t)a.n_requests * a.beams * beam_chunks(a.vocab);
    uint64_t o = 0;
    auto take = [&](uint64_t bytes) { uint64_t r = o; o = (o + bytes + 255) & ~uint64_t(255); return r; };
    if (a.beams * beam_chunks(a.vocab) <= FUSED_UNITS) return 0;
    const uint64_t s = take(units * 8), m = take(units * 4), l = take(units * a.beams * 8);
    if (w) {
        char* p = (char*)a.workspace;
        w->sum = (double*)(p + s); w->max = (float*)(p + m); w->list = (float2*)(p + l);
    }
    return o;
}

// Best first: larger value, then lower index.
// (An int, combined with & so that no step becomes a branch.)
__device__ __forceinline__ int before(float va, int ia, float vb, int ib) {
    return (int)(va > vb) | ((int)(va == vb) & (int)(ia < ib));
}

__device__ __forceinline__ float min_f(float a, float b) { return a < b ? a : b; }

// One wave: chunk `ch` of row `row`; list[0 .. beams) gets its best logits
// (-infinity and the last index behind what the chunk has), mx and sum its
// normaliser's part.  buf: CAP entries of LDS of this wave.
__device__ __forceinline__ void beam_chunk(const mtp_beam_args& a, int row, int ch, float2* list, float* mx_out,
                                           double* sum_out, float2* buf) {
    const int lane = threadIdx.x & 63, W = a.beams;
    const float* x = a.logits + (int64_t)row * a.ld;
    const int v0 = ch * CHUNK + lane;
    const int hide = a.len[row] < a.eos_min ? a.eos_id : -1;
    float f[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = v0 + 64 * i;
        f[i] = v < a.vocab ? x[v] : -INFINITY;
    }
    if (hide / CHUNK == ch) {                    // (uniform; -1 / CHUNK is 0: no index is -1)
#pragma unroll
        for (int i = 0; i < NV; ++i) f[i] = v0 + 64 * i == hide ? -INFINITY : f[i];
    }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        f[i] = fmaxf(f[i], -INFINITY);           // NaN: -infinity
        top = fmaxf(top, f[i]);
    }
    // a bound that at least W of the chunk's logits reach: the W-th largest of the lanes' maxima, or (fewer instructions,
    // more logits that reach it) the smallest maximum of at least W groups of lanes
    float bound;
    if (W > FEW_BEAMS) {
        int above = 0;
#pragma unroll
        for (int k = 0; k < 64; ++k) above += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(top), k)) > top ? 1 : 0;
        bound = above < W ? top : INFINITY;
        bound = min_f(bound, dpp_f<DPP_XOR1>(bound));
    } else {
        bound = fmaxf(top, dpp_f<DPP_XOR1>(top));
        bound = fmaxf(bound, dpp_f<DPP_XOR2>(bound));
        bound = fmaxf(bound, dpp_f<DPP_HALF_MIRROR>(bound));
        bound = fmaxf(bound, dpp_f<DPP_ROR8>(bound));
    }
    bound = min_f(bound, dpp_f<DPP_XOR2>(bound));
    bound = min_f(bound, dpp_f<DPP_HALF_MIRROR>(bound));
    bound = min_f(bound, dpp_f<DPP_ROR8>(bound));
    float other, mine = pl_lo16(bound, other);
    bound = min_f(mine, other);
    mine = pl_lo32(bound, other);
    bound = min_f(mine, other);
    const float m = wave_max64(top);
    // float32 exponentials, summed in float64 (16 requests of 8 beams over 65,536 logits 20.6 us; 20.3 us with float32
    // sums of eight, which lose what is below 2^-24 of the largest); a chunk without a finite logit adds 0
    const float mm = m == -INFINITY ? 0.f : m;
    double part[4] = {0.0, 0.0, 0.0, 0.0};       // (four chains of additions)
#pragma unroll
    for (int i = 0; i < NV; ++i) part[i & 3] += (double)__builtin_amdgcn_exp2f((f[i] - mm) * LOG2E);
    double sum = (part[0] + part[1]) + (part[2] + part[3]);
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) { *mx_out = m; *sum_out = sum; }

    if (__any(bound == -INFINITY)) {
        // nothing behind the vocabulary reaches it (4 requests of 11 beams over 2057 logits 16.4 us, 30.7 us with all of
        // the last chunk gathered)
#pragma unroll
        for (int i = 0; i < NV; ++i) f[i] = v0 + 64 * i < a.vocab ? f[i] : NAN;
    }
    int n = 0;                                   // uniform
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint64_t hit = __ballot(f[i] >= bound);
        if (hit) {
            const int at = n + __popcll(hit & ((1ull << lane) - 1));
            if (f[i] >= bound && at < CAP) buf[at] = make_float2(f[i], __int_as_float(v0 + 64 * i));
            n += __popcll(hit);
        }
    }
    __builtin_amdgcn_wave_barrier();
    if (n <= 64) {
        // a lane each: its place is the number of candidates before it
        const float2 e = buf[lane < n ? lane : 0];
        const int id = __float_as_int(e.y);
        int place = 0;
        for (int k = 0; k < n; ++k) {
            const float v = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(e.x), k));
            place += before(v, __builtin_amdgcn_readlane(id, k), e.x, id);
        }
        if (lane < n && place < W) list[place] = e;
        if (lane >= n && lane < W) list[lane] = make_float2(-INFINITY, __int_as_float(0x7fffffff));
        return;
    }
    float pv = INFINITY;                         // the last one taken
    int pi = -1;
    if (n <= CAP) {
        float cv[CAP / 64];
        int ci[CAP / 64];
#pragma unroll
        for (int k = 0; k < CAP / 64; ++k) {
            const bool in = 64 * k + lane < n;
            const float2 e = buf[in ? 64 * k + lane : 0];
            cv[k] = in ? e.x : -INFINITY;
            ci[k] = in ? __float_as_int(e.y) : 0x7fffffff;
        }
        for (int w = 0; w < W; ++w) {
            float bv = -INFINITY;
            int bi = 0x7fffffff;
#pragma unroll
            for (int k = 0; k < CAP / 64; ++k)
                if (before(pv, pi, cv[k], ci[k]) & before(cv[k], ci[k], bv, bi)) { bv = cv[k]; bi = ci[k]; }
            wave_argmax_uniform(bv, bi);
            if (lane == 0) list[w] = make_float2(bv, __int_as_float(bi));
            pv = bv; pi = bi;
        }
    } else {
        // many equal logits: all of the chunk, once per place
        for (int w = 0; w < W; ++w) {
            float bv = -INFINITY;
            int bi = 0x7fffffff;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (before(pv, pi, f[i], v0 + 64 * i) & before(f[i], v0 + 64 * i, bv, bi)) { bv = f[i]; bi = v0 + 64 * i; }
            wave_argmax_uniform(bv, bi);
            if (lane == 0) list[w] = make_float2(bv, __int_as_float(bi));
            pv = bv; pi = bi;
        }
    }
}

// The waves' own scratch.
struct BeamLds {
    double lse[MAX_BEAMS], den[MAX_BEAMS];
    float score[MAX_BEAMS];
    int len[MAX_BEAMS], done[MAX_BEAMS];
    float2 best[MAX_BEAMS][MAX_BEAMS];           // each beam's best logits over its chunks
    double rank[MAX_BEAMS][MAX_BEAMS];           // its candidates, best first
    int place[PLACED * PLACED];                  // each candidate's place among all
    int win[MAX_BEAMS];                          // the chosen: beam * MAX_BEAMS + place in its list
};

// The id of the largest value among lanes 0 .. W - 1 (W <= 32), of equal
// ones the lowest; uniform.
__device__ __forceinline__ int best_head(double v, int id, int W) {
    auto take = [&](double ov, int oi) {
        const bool better = (int)(ov > v) | ((int)(ov == v) & (int)(oi < id));
        v = better ? ov : v;
        id = better ? oi : id;
    };
    auto join = [](int lo, int hi) { return __longlong_as_double((long long)(uint32_t)lo | (long long)hi << 32); };
#define STEP(CTRL) take(join(dpp_i<CTRL>(__double2loint(v)), dpp_i<CTRL>(__double2hiint(v))), dpp_i<CTRL>(id))
    STEP(DPP_XOR1);
    STEP(DPP_XOR2);
    STEP(DPP_HALF_MIRROR);
    if (W > 8) STEP(DPP_ROR8);
#undef STEP
    if (W > 16) {
        const double ov = join(__builtin_amdgcn_readlane(__double2loint(v), 16), __builtin_amdgcn_readlane(__double2hiint(v), 16));
        take(ov, __builtin_amdgcn_readlane(id, 16));
    }
    return __builtin_amdgcn_readfirstlane(id);
}

// The request's state, by the workgroup's last wave (read after a barrier).
template <int NW>
__device__ __forceinline__ void beam_state(const mtp_beam_args& a, int r, BeamLds& s) {
    const int b = (int)threadIdx.x - 64 * (NW - 1);
    if (b < 0 || b >= a.beams) return;
    const int row = r * a.beams + b, dn = a.done[row] > 0, len = a.len[row] + (dn ? 0 : 1);
    s.done[b] = dn; s.len[b] = len; s.score[b] = a.score[row];
    s.den[b] = a.alpha == 0.f ? 1.0 : pow((double)max(len, 1), (double)a.alpha);
}

// A request's merge by a workgroup of NW waves.  max, sum, list: the request's
// own, [beams][chunks] and [beams][chunks][beams].  held: room for HOLD entries of
// this wave's, into which it takes a beam's lists that fit; HOLD 0: they are in
// LDS already.
template <int NW, int HOLD>
__device__ __forceinline__ void beam_merge(const mtp_beam_args& a, int r, const float* max, const double* sum,
                                           const float2* list, int chunks, BeamLds& s, float2* held) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, W = a.beams, n = min(W, a.vocab);
    for (int b = wave; b < W; b += NW) {
        if (a.done[r * W + b] > 0) continue;     // uniform over the wave
        const float2* bl = list + (size_t)b * chunks * W;
        const int entries = chunks * W;
        const bool holds = HOLD > 0 && entries <= HOLD;
        constexpr int PRE = HOLD <= 256 ? HOLD / 64 : 0;      // of a lane in flight during the sums below (more would spill)
        float2 pre[PRE + 1];
        if (holds) {
#pragma unroll
            for (int i = 0; i < PRE; ++i) pre[i] = bl[min(64 * i + lane, entries - 1)];
        }
        const float* bm = max + (size_t)b * chunks;
        const double* bs = sum + (size_t)b * chunks;
        float m = -INFINITY;
        for (int i = lane; i < chunks; i += 64) m = fmaxf(m, bm[i]);
        m = wave_max64(m);
        double t = 0.0;
        for (int i = lane; i < chunks; i += 64) t += bs[i] * exp((double)bm[i] - (double)m);
        for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o);
        if (lane == 0) s.lse[b] = (double)m + log(t);
        if (chunks == 1) {
            if (lane < n) s.best[b][lane] = bl[lane];
            continue;
        }
        const float2* src = bl;
        if (holds) {
            __builtin_amdgcn_wave_barrier();     // (the last beam's are read)
#pragma unroll
            for (int i = 0; i < PRE; ++i)
                if (64 * i + lane < entries) held[64 * i + lane] = pre[i];
            for (int i = 64 * PRE + lane; i < entries; i += 64) held[i] = bl[i];
            __builtin_amdgcn_wave_barrier();
            src = held;
        }
        if (chunks <= 64) {
            // lane i: the head of chunk i's list
            const float2 none = make_float2(-INFINITY, __int_as_float(0x7fffffff));
            int pos = 0;
            float2 head = lane < chunks ? src[lane * W] : none;
            for (int w = 0; w < n; ++w) {
                float bv = head.x;
                int bi = __float_as_int(head.y);
                wave_argmax_uniform(bv, bi);
                if (lane == 0) s.best[b][w] = make_float2(bv, __int_as_float(bi));
                if (__float_as_int(head.y) == bi) head = ++pos < W ? src[lane * W + pos] : none;
            }
            continue;
        }
        // lane i: the heads of the lists of chunks i, i + 64, ... (the best of them, advanced past what was taken)
        float pv = INFINITY;
        int pi = -1;
        float hv = -INFINITY;
        int hi = 0x7fffffff;
        bool stale = true;
        for (int w = 0; w < n; ++w) {
            if (stale) {
                hv = -INFINITY; hi = 0x7fffffff;
                for (int i = lane; i < chunks; i += 64)
                    for (int k = 0; k < W; ++k) {
                        const float2 e = src[(size_t)i * W + k];
                        const int id = __float_as_int(e.y);
                        if (before(pv, pi, e.x, id)) {
                            if (before(e.x, id, hv, hi)) { hv = e.x; hi = id; }
                            break;
                        }
                    }
            }
            float bv = hv;
            int bi = hi;
            wave_argmax_uniform(bv, bi);
            if (lane == 0) s.best[b][w] = make_float2(bv, __int_as_float(bi));
            stale = hi == bi;
            pv = bv; pi = bi;
        }
    }
    __syncthreads();
    // the candidates, W lists of n: a finished beam's are itself and then the tokens that it cannot take, those of a
    // beam without a finite score or normaliser all -infinity, in token order
    auto candidate = [&](int b, int j, int& tok) {
        double total = -INFINITY;
        if (!(fabsf(s.score[b]) < INFINITY)) {
            tok = j;
        } else if (s.done[b]) {
            tok = j == 0 ? a.eos_id : (j - 1 < a.eos_id ? j - 1 : j);
            if (j == 0) total = (double)s.score[b];
        } else if (!(fabs(s.lse[b]) < INFINITY)) {
            tok = j;
        } else {
            tok = __float_as_int(s.best[b][j].y);
            total = (double)s.score[b] + ((double)s.best[b][j].x - s.lse[b]);
        }
        return total;
    };
    for (int c = threadIdx.x; c < W * n; c += 64 * NW) {
        const int b = c / n, j = c - b * n;
        int tok;
        s.rank[b][j] = candidate(b, j, tok) / s.den[b];
        if (W <= PLACED) s.place[c] = j;
    }
    __syncthreads();
    if (W > PLACED) {
        // the best of the lists' heads, W times; equal ones: the earlier beam's
        if (wave == 0) {
            int pos = 0, id = lane < W ? lane : 64 + lane;
            double head = lane < W ? s.rank[lane][0] : -INFINITY;
            for (int w = 0; w < W; ++w) {
                const int best = best_head(head, id, W);
                if (id != best) continue;
                s.win[w] = lane * MAX_BEAMS + pos++;
                head = pos < n ? s.rank[lane][pos] : -INFINITY;
                id = pos < n ? lane : 64 + lane;
            }
        }
    } else {
        // a candidate's place: those of its own beam before it, and how many of every other beam's come before it
        // (equal ones: those of the earlier beam)
        for (int p = threadIdx.x; p < W * n * W; p += 64 * NW) {
            const int c = p / W, o = p - c * W, b = c / n, j = c - b * n;
            if (o == b) continue;
            const double mine = s.rank[b][j];
            int lo = 0, hi = n;
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                const double r2 = s.rank[o][mid];
                if (r2 > mine || (r2 == mine && o < b)) lo = mid + 1; else hi = mid;
            }
            if (lo) atomicAdd(&s.place[c], lo);
        }
        __syncthreads();
        for (int c = threadIdx.x; c < W * n; c += 64 * NW)
            if (s.place[c] < W) s.win[s.place[c]] = c / n * MAX_BEAMS + c % n;
    }
    __syncthreads();
    for (int w = threadIdx.x; w < W; w += 64 * NW) {
        const int b = s.win[w] / MAX_BEAMS, j = s.win[w] % MAX_BEAMS, o = r * W + w;
        int tok;
        const double total = candidate(b, j, tok);
        a.out_score[o] = (float)total;
        a.out_len[o] = s.len[b];
        a.out_done[o] = s.done[b] | (tok == a.eos_id ? 1 : 0);
        a.out_parent[o] = r * W + b;
        a.out_token[o] = tok;
    }
}

// One launch per request: few chunks.
template <int NW>
__global__ __launch_bounds__(64 * NW) void beam_fused_kernel(mtp_beam_args a) {
    __shared__ BeamLds s;
    __shared__ float2 s_buf[NW][CAP], s_list[FUSED_UNITS * MAX_BEAMS];
    __shared__ float s_max[FUSED_UNITS];
    __shared__ double s_sum[FUSED_UNITS];
    const int r = blockIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), W = a.beams;
    const int chunks = (a.vocab + CHUNK - 1) / CHUNK;
    beam_state<NW>(a, r, s);
    for (int u = wave; u < W * chunks; u += NW) {
        const int b = u / chunks;
        if (a.done[r * W + b] > 0) continue;
        beam_chunk(a, r * W + b, u - b * chunks, s_list + u * W, &s_max[u], &s_sum[u], s_buf[wave]);
    }
    __syncthreads();
    beam_merge<NW, 0>(a, r, s_max, s_sum, s_list, chunks, s, nullptr);
}

__global__ __launch_bounds__(256) void beam_chunk_kernel(mtp_beam_args a, BeamWs w, int chunks) {
    __shared__ float2 s_buf[4][CAP];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = blockIdx.y, ch = blockIdx.x * 4 + wave;
    if (ch >= chunks || a.done[row] > 0) return;
    const size_t u = (size_t)row * chunks + ch;
    beam_chunk(a, row, ch, w.list + u * a.beams, &w.max[u], &w.sum[u], s_buf[wave]);
}

template <int NW, int HOLD>
__global__ __launch_bounds__(64 * NW) void beam_merge_kernel(mtp_beam_args a, BeamWs w, int chunks) {
    __shared__ BeamLds s;
    __shared__ float2 s_held[NW][HOLD];
    const size_t u = (size_t)blockIdx.x * a.beams * chunks;
    beam_state<NW>(a, blockIdx.x, s);
    beam_merge<NW, HOLD>(a, blockIdx.x, w.max + u, w.sum + u, w.list + u * a.beams, chunks, s, s_held[threadIdx.x >> 6]);
}

// ------------------------------------------------- a context's beams
__global__ __launch_bounds__(256) void beam_prepare_kernel(BeamRowsArgs a) {
    const int b = blockIdx.x * 256 + threadIdx.x;
    if (b >= a.B) return;
    const int n = a.out_cnt[b];                  // a row that had ended before the step emitted nothing
    a.len[b] = a.st[b].gen - n;
    a.done[b] = n == 0 ? 1 : 0;
    a.ctx[b] = a.st[b].ctx_len;
    if (a.fresh) a.score[b] = b % a.beams == 0 ? 0.f : -INFINITY;
}

// Row c as its parent's continuation by its token.
__global__ __launch_bounds__(256) void beam_follow_kernel(BeamRowsArgs a) {
    const int c = blockIdx.x, p = a.parent[c], ended = a.done[p], tok = a.token[c];
    SeqState s = a.st[p];
    const int g = a.len[p];
    const int32_t* from = a.hist + (size_t)p * a.max_new;
    int32_t* to = a.new_hist + (size_t)c * a.max_new;
    for (int i = threadIdx.x; i < g; i += 256) to[i] = from[i];
    if (threadIdx.x != 0) return;
    if (!ended) {
        to[g] = tok;
        const bool done = tok == a.eos_id || g + 1 >= a.max_new;
        s.gen = g + 1;
        s.done = done ? 1 : 0;
        s.pend_len = done ? 0 : 1;
        s.pend_ids[0] = tok;
        s.last_tok = tok;
    }
    a.add[c] = s.prompt_len + a.max_new - s.ctx_len;
    a.out_tok[c] = ended ? -1 : tok;
    a.out_cnt[c] = ended ? 0 : 1;
    a.new_st[c] = s;
}

__global__ __launch_bounds__(256) void beam_apply_kernel(BeamRowsArgs a) {
    const int c = blockIdx.x;
    const SeqState s = a.new_st[c];
    for (int i = threadIdx.x; i < s.gen; i += 256) a.hist[(size_t)c * a.max_new + i] = a.new_hist[(size_t)c * a.max_new + i];
    // (unused table entries name page 0, so that loads past the context stay in the pool)
    for (int i = threadIdx.x; i < a.maxp; i += 256) a.btab[(size_t)c * a.maxp + i] = max(0, a.new_tab[(size_t)c * a.maxp + i]);
    if (threadIdx.x == 0) a.st[c] = s;
}

bool aligned(const void* p, uintptr_t n) { return p && ((uintptr_t)p & (n - 1)) == 0; }

int beam_check(const mtp_beam_args* a) {
    if (!a) return MTP_EINVAL;
    if (a->beams < 1 || a->beams > MAX_BEAMS || a->n_requests < 0 || (int64_t)a->n_requests * a->beams > 65535 ||
        a->vocab < 1 || a->vocab >= (1 << 24) || a->eos_id < 0 || a->eos_id >= a->vocab || !(a->alpha >= 0.f) ||
        a->alpha > 32.f)                         // (2^31)^32 is a finite float64
        return MTP_EINVAL;
    return MTP_OK;
}

}  // namespace
hipError_t beam_rows_prepare(hipStream_t st, const BeamRowsArgs& a) {
    hipLaunchKernelGGL(beam_prepare_kernel, dim3((a.B + 255) / 256), dim3(256), 0, st, a);
    return hipGetLastError();
}
hipError_t beam_rows_follow(hipStream_t st, const BeamRowsArgs& a) {
    hipLaunchKernelGGL(beam_follow_kernel, dim3(a.B), dim3(256), 0, st, a);
    return hipGetLastError();
}
hipError_t beam_rows_apply(hipStream_t st, const BeamRowsArgs& a) {
    hipLaunchKernelGGL(beam_apply_kernel, dim3(a.B), dim3(256), 0, st, a);
    return hipGetLastError();
}

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
        !aligned(a.out_token, 4) || a.ld < a.vocab)
        return MTP_EINVAL;
    BeamWs w{};
    const uint64_t need = beam_carve(a, &w);
    if (need && !aligned(a.workspace, 256)) return MTP_EINVAL;
    if (need > a.workspace_bytes) return MTP_ENOMEM;
    hipStream_t st = (hipStream_t)hip_stream;
    const int chunks = beam_chunks(a.vocab);
    if (need == 0) {
        if (a.beams * chunks <= 4) hipLaunchKernelGGL(beam_fused_kernel<4>, dim3(a.n_requests), dim3(256), 0, st, a);
        else hipLaunchKernelGGL(beam_fused_kernel<16>, dim3(a.n_requests), dim3(1024), 0, st, a);
    } else {
        hipLaunchKernelGGL(beam_chunk_kernel, dim3((chunks + 3) / 4, a.n_requests * a.beams), dim3(256), 0, st, a, w, chunks);
        if (a.beams * chunks <= 256)
            hipLaunchKernelGGL((beam_merge_kernel<16, 256>), dim3(a.n_requests), dim3(1024), 0, st, a, w, chunks);
        else
            hipLaunchKernelGGL((beam_merge_kernel<16, 1024>), dim3(a.n_requests), dim3(1024), 0, st, a, w, chunks);
    }
    return hipGetLastError() == hipSuccess ? MTP_OK : MTP_EHIP;
}

}  // extern "C"
