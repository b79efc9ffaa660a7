// Verification of drafted tokens against the target's probabilities
// (mtp_verify_drafts).  See include/mtp.h for the operator's definition.
//
//   p(v) = exp((x[v] - M) / T) / Z,  Z = sum_v exp((x[v] - M) / T),  M = max x
//   accept draft d iff u q(d) < p(d); else draw v by max(p(v) - q(v), 0)
//
// A drawn token is a whole number that must not depend on the order of a sum:
// with float32 exponentials the borders of 65,536 tokens' shares are each off by
// some 10^-8 of the whole, which moves a draw in a thousand.  Exponentials and
// sums are float64 (borders within 10^-14).
//
// One wave takes a chunk of 512 or 1024 logits into registers and leaves its maximum
// and sum; a row's workgroup then joins its tokens' chunks, judges its drafts, finds
// the drawn token's chunk by the chunks' shares and the token in it by a scan.  The
// shares of p are the chunks' sums over again; a refused certain draft takes a pass
// over its own chunk, and max(p - q, 0) one over the refused draft's two rows, by a
// wave a chunk.
//
// What bounds it: of few logits the chain lengths -> logits -> sums -> drafts -> the
// drawn chunk -> its logits (4 tokens of 1025 logits 8.8 us; 64 rows of up to 8, 11.2
// us).  Of many the float64 pipe and the loads in turn (32 rows of up to 8 tokens over
// 65,536 logits, 76 MB with draft logits: the chunks 22.3 us at 3.4 TB/s with the pipe
// busy half the time; two or four chunks a wave one after another, the next one's loads
// ahead, took 1 to 6 us longer), then two such chains (8.9 us and 7.0 us).
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <limits>

#include "../../include/mtp.h"
#include "common.h"
#include "wave.h"

namespace mtp {
namespace {

constexpr int MAX_WIDTH = 256;
constexpr int NW = 16;                           // waves of a row's workgroup
constexpr int WIDE_NV = 16;                      // logits of a lane in a chunk, where it is not 8
constexpr int EACH = 8;                          // logits of a lane where a drawn token is looked for
// Up to this many chunks of 512 of a row's tokens (and draft rows) one launch does everything.  Whole calls in one launch and in
// two: 16 rows of 4 tokens of 1025 logits, 12 chunks, 9.5 and 10.8 us, of 8 tokens, 24, 10.9 and 10.8, of 10, 30, 12.2 and 11.1,
// of 16, 48, 14.4 and 11.2; 64 rows, 24 chunks, 11.1 and 11.3, 30, 12.3 and 11.7; one row, 12, 9.1 and 10.0, 24, 10.4 and 10.1
// (three launches, draft logits, 24 chunks: 11.7 and 12.4; 32: 12.3 either way).  256 rows are faster in one at every number measured,
// 96 at most (48 chunks 15.2 and 19.7).
constexpr int FUSED_UNITS = 24;

// A chunk's, or a row's: its largest logit, the sum of exp((x - max) / T), and with
// temperature 0 the first place of the largest.
struct Stat {
    double sum;
    float max;
    int at;
};

// What a row's drafts came to: the token whose logits are drawn from, and how.
struct Judged {
    double pz, qz;                               // 1 / Z of its two distributions, and below their largest logits
    float pm, qm;
    int at;                                      // (temperature 0) the place of the largest
    int t, i;                                    // the token, its place in the row; i < 0: nothing to draw
    int accepted, refused, draft;                // whether a draft was refused, and which
    int live, done;                              // accepted drafts up to the first end; there is one
};

struct VerifyWs {
    Stat* stat;                                  // [rows * width][1 or 2][chunks]
    double* mass;                                // [rows][chunks of 512] shares of max(p - q, 0)
    Judged* judged;                              // [rows]
};

// Chunks of a vocabulary with nv logits a lane.
__host__ __device__ __forceinline__ int chunks_of(int vocab, int nv) { return (vocab + 64 * nv - 1) / (64 * nv); }

// 2^z for z <= 0: z = k + r, |r| <= 1/2; 1 + r q(r) of degree 10, q through (2^r - 1) / r at the ten Chebyshev points of
// [-1/2, 1/2] (2^r to 2^-50.6 of itself, 1 at 0), its exponent field k higher.  From -1023 down it is +0: the field's end.
// (With e^z by the Taylor polynomial to z^11 between rint and ldexp: 32 rows of up to 8 tokens over 65,536 logits, the
// chunks alone, 28.7 us; 23.0 us.)
__device__ __forceinline__ double exp2_neg(double z) {
    constexpr double ROUND = 6755399441055744.0;                       // 1.5 x 2^52: sums with it are whole
    z = fmax(z, -1023.0);
    const double t = z + ROUND, r = z - (t - ROUND);
    double e = 7.070977866508138e-09;
    e = fma(e, r, 1.0205905413765595e-07);
    e = fma(e, r, 1.3215451633221434e-06);
    e = fma(e, r, 1.5252672924850737e-05);
    e = fma(e, r, 0.00015403530424776529);
    e = fma(e, r, 0.0013333558200794592);
    e = fma(e, r, 0.009618129107618665);
    e = fma(e, r, 0.05550410866465167);
    e = fma(e, r, 0.24022650695910075);
    e = fma(e, r, 0.6931471805599462);
    e = fma(e, r, 1.0);
    return __hiloint2double(__double2hiint(e) + (__double2loint(t) << 20), __double2loint(e));
}
// exp((x - m) / T) for x <= m, with scale = log2(e) / T; infinite logits share the whole, rows of -infinity hold nothing.
__device__ __forceinline__ double rel(float x, float m, double scale) {
    const double e = exp2_neg(((double)x - (double)m) * scale);
    return x == m ? (m == -INFINITY ? 0.0 : 1.0) : e;
}

template <int CTRL>
__device__ __forceinline__ double dpp_d(double v) {
    const int lo = dpp_i<CTRL>(__double2loint(v)), hi = dpp_i<CTRL>(__double2hiint(v));
    return __longlong_as_double((long long)(uint32_t)lo | (long long)hi << 32);
}
__device__ __forceinline__ double join_d(uint32_t lo, uint32_t hi) {
    return __longlong_as_double((long long)lo | (long long)hi << 32);
}
// The same sum on every lane.
__device__ __forceinline__ double wave_sum_d(double v) {
    v += dpp_d<DPP_XOR1>(v);
    v += dpp_d<DPP_XOR2>(v);
    v += dpp_d<DPP_HALF_MIRROR>(v);
    v += dpp_d<DPP_ROR8>(v);
    auto lo = __builtin_amdgcn_permlane16_swap(__double2loint(v), __double2loint(v), false, false);
    auto hi = __builtin_amdgcn_permlane16_swap(__double2hiint(v), __double2hiint(v), false, false);
    v = join_d(lo[0], hi[0]) + join_d(lo[1], hi[1]);
    lo = __builtin_amdgcn_permlane32_swap(__double2loint(v), __double2loint(v), false, false);
    hi = __builtin_amdgcn_permlane32_swap(__double2hiint(v), __double2hiint(v), false, false);
    return join_d(lo[0], hi[0]) + join_d(lo[1], hi[1]);
}
// The sum over the lanes up to each.
__device__ __forceinline__ double wave_run_d(double v) {
    const int lane = threadIdx.x & 63;
    for (int o = 1; o < 64; o <<= 1) {
        const double y = __shfl_up(v, o);
        if (lane >= o) v += y;
    }
    return v;
}

// A row's token range and the id that its token i hides (-1: none).
struct Row { int s, n; };
__device__ __forceinline__ Row row_of(const mtp_verify_args& a, int r) {
    const int s = max(0, min(a.row_start[r], a.n_tokens)), e = max(s, min(a.row_start[r + 1], a.n_tokens));
    return Row{s, min(e - s, a.width)};
}
__device__ __forceinline__ int hidden(const mtp_verify_args& a, int r, int i) {
    return a.eos_id >= 0 && a.eos_min > 0 && (int64_t)a.len[r] + i < a.eos_min ? a.eos_id : -1;
}
// Logit x of token v as it counts; NaN: -infinity.
__device__ __forceinline__ float shown(float x, int v, int hide) { return v == hide ? -INFINITY : fmaxf(x, -INFINITY); }

// Chunk ch of the logits x by a wave.
template <bool GREEDY, int NV>
__device__ __forceinline__ Stat chunk_stat(const float* x, int vocab, int ch, int hide, double scale) {
    constexpr int CHUNK = 64 * NV;
    const int lane = threadIdx.x & 63, v0 = ch * CHUNK + lane;
    float f[NV];
    if ((ch + 1) * CHUNK <= vocab) {                                   // uniform
#pragma unroll
        for (int i = 0; i < NV; ++i) f[i] = x[v0 + 64 * i];
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) f[i] = x[min(v0 + 64 * i, vocab - 1)];
#pragma unroll
        for (int i = 0; i < NV; ++i) f[i] = v0 + 64 * i < vocab ? f[i] : -INFINITY;
    }
    if (hide >= 0 && hide / CHUNK == ch) {                             // uniform
#pragma unroll
        for (int i = 0; i < NV; ++i) f[i] = v0 + 64 * i == hide ? -INFINITY : f[i];
    }
    // (NaN are never larger, and their exponentials come to 0)
    Stat s{0.0, -INFINITY, 0x7fffffff};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (GREEDY && f[i] > s.max) s.at = v0 + 64 * i;
        s.max = fmaxf(s.max, f[i]);
    }
    if (GREEDY) {
        wave_argmax(s.max, s.at);
        return s;
    }
    s.max = wave_max64(s.max);
    double part[4] = {0.0, 0.0, 0.0, 0.0};
    if (fabsf(s.max) < INFINITY) {                                     // uniform
        const double m = s.max;
#pragma unroll
        for (int i = 0; i < NV; ++i) part[i & 3] += exp2_neg(((double)f[i] - m) * scale);
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) part[0] += f[i] == INFINITY ? 1.0 : 0.0;
    }
    s.sum = wave_sum_d((part[0] + part[1]) + (part[2] + part[3]));
    return s;
}

// A row's chunks joined, by a wave.
template <bool GREEDY>
__device__ __forceinline__ Stat join_stat(const Stat* c, int chunks, double scale) {
    const int lane = threadIdx.x & 63;
    Stat s{0.0, -INFINITY, 0x7fffffff};
    for (int i = lane; i < chunks; i += 64) {
        const float m = c[i].max;
        if (GREEDY && (m > s.max || (m == s.max && c[i].at < s.at))) s.at = c[i].at;
        s.max = fmaxf(s.max, m);
    }
    if (GREEDY) {
        wave_argmax(s.max, s.at);
        return s;
    }
    s.max = wave_max64(s.max);
    for (int i = lane; i < chunks; i += 64) s.sum += c[i].sum * rel(c[i].max, s.max, scale);
    s.sum = wave_sum_d(s.sum);
    return s;
}

// LDS of a row's workgroup.
struct RowLds {
    Stat p[MAX_WIDTH], q[MAX_WIDTH];
    double px[MAX_WIDTH];                        // the target's probability of the draft behind token i
    int ok[MAX_WIDTH];                           // bit 0: it is accepted; bit 1: it is the end
    int draft[MAX_WIDTH];
    double own, run[EACH];                       // the refused draft's chunk; the pick's waves
    int found[2][EACH];
};

// The draft behind a row's token i (-1: none, or outside the vocabulary), its logits and its uniform.
struct Draft {
    int d;
    float x, y, u;
};
// Of the i that the thread judges, from the last thread down: loaded ahead, while the row's first waves have chunks to do.
template <bool GREEDY, bool DRAWN, int W>
__device__ __forceinline__ Draft draft_of(const mtp_verify_args& a, const Row& row) {
    static_assert(64 * W >= MAX_WIDTH, "a thread a token");
    const int i = 64 * W - 1 - (int)threadIdx.x, t = row.s + i;
    Draft m{-1, 0.f, 0.f, 0.f};
    if (i + 1 < row.n) {
        m.d = a.tokens[t + 1];
        m.u = a.uniforms[t + 1];
        if (!GREEDY) {
            const int d = max(0, min(m.d, a.vocab - 1));
            m.x = a.logits[(int64_t)t * a.ld + d];
            if (DRAWN) m.y = a.draft[(int64_t)t * a.draft_ld + d];
        }
    }
    return m;
}

// The drafts of row r by a workgroup of W waves; stat: the row's chunks.  Every thread gets the result.
template <bool GREEDY, bool DRAWN, int W>
__device__ __forceinline__ Judged judge(const mtp_verify_args& a, int r, const Row& row, const Draft& mine, const Stat* stat,
                                        int chunks, double scale, RowLds& s) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int PER = DRAWN ? 2 : 1;
    for (int u = wave; u < row.n * PER; u += W) {
        const int i = u / PER, which = u - i * PER;
        if (which && i + 1 >= row.n) continue;
        const Stat v = join_stat<GREEDY>(stat + (size_t)u * chunks, chunks, scale);
        if (lane == 0) (which ? s.q : s.p)[i] = v;
    }
    __syncthreads();
    const int i = 64 * W - 1 - (int)threadIdx.x;
    if (i < row.n) {
        const int hide = hidden(a, r, i);
        bool ok = false;
        double px = 0.0;
        if (mine.d >= 0 && mine.d < a.vocab) {
            const Stat p = s.p[i];
            if (GREEDY) {
                ok = p.max > -INFINITY && p.at == mine.d;
                px = ok ? 1.0 : 0.0;
            } else if (p.sum > 0.0) {
                px = rel(shown(mine.x, mine.d, hide), p.max, scale) / p.sum;
                double qx = 1.0;
                if (DRAWN) {
                    const Stat q = s.q[i];
                    qx = q.sum > 0.0 ? rel(shown(mine.y, mine.d, hide), q.max, scale) / q.sum : 0.0;
                }
                ok = (double)mine.u * qx < px;
            }
        }
        s.px[i] = px;
        s.draft[i] = mine.d;
        s.ok[i] = (ok ? 1 : 0) | (i + 1 < row.n && mine.d == a.eos_id ? 2 : 0);
    }
    __syncthreads();
    Judged j;
    j.accepted = j.live = j.done = 0;
    while (j.accepted + 1 < row.n && (s.ok[j.accepted] & 1)) {
        j.live += j.done ? 0 : 1;
        j.done |= s.ok[j.accepted++] >> 1;
    }
    // (a row of -infinity alone gives no token)
    const bool any = row.n > 0 && !j.done && s.p[j.accepted].max > -INFINITY;
    j.i = any ? j.accepted : -1;
    j.t = row.s + j.accepted;
    j.refused = j.accepted + 1 < row.n ? 1 : 0;
    j.draft = j.refused ? s.draft[j.accepted] : -1;
    j.pz = j.qz = 0.0;
    j.pm = j.qm = 0.f;
    j.at = 0;
    if (any) {
        const Stat p = s.p[j.accepted];
        j.pm = p.max;
        j.pz = GREEDY ? 1.0 : 1.0 / p.sum;
        j.at = p.at;
        if (DRAWN && j.refused) {
            const Stat q = s.q[j.accepted];
            j.qm = q.max;
            j.qz = q.sum > 0.0 ? 1.0 / q.sum : 0.0;
        }
    }
    return j;
}

// The share of token v in what a judged row's draw takes: p, without the refused draft, or max(p - q, 0).
template <bool DRAWN>
__device__ __forceinline__ double share(const mtp_verify_args& a, const Judged& j, float x, float y, int v, double scale) {
#pragma clang fp contract(off)                   // (equal p and q leave 0, which a fused product would not)
    const double p = rel(x, j.pm, scale) * j.pz;
    if (!j.refused) return p;
    if (!DRAWN) return v == j.draft ? 0.0 : p;
    const double q = rel(y, j.qm, scale) * j.qz;
    return fmax(p - q, 0.0);
}

// Chunk ch's share of what is drawn, by a wave.
template <bool DRAWN, int NV>
__device__ __forceinline__ double chunk_mass(const mtp_verify_args& a, const Judged& j, int hide, int ch, double scale) {
    const int v0 = ch * 64 * NV + (threadIdx.x & 63);
    const float *xp = a.logits + (int64_t)j.t * a.ld, *yp = DRAWN ? a.draft + (int64_t)j.t * a.draft_ld : xp;
    float x[NV], y[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = min(v0 + 64 * i, a.vocab - 1);
        x[i] = xp[v];
        if (DRAWN) y[i] = yp[v];
    }
    double part[2] = {0.0, 0.0};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = v0 + 64 * i;
        const float fx = shown(x[i], v, hide), fy = DRAWN ? shown(y[i], v, hide) : 0.f;
        const double m = share<DRAWN>(a, j, fx, fy, v, scale);
        part[i & 1] += v < a.vocab ? m : 0.0;
    }
    return wave_sum_d(part[0] + part[1]);
}

// The whole of the chunks' shares mass(c), the same on every lane of every wave.
template <typename F>
__device__ __forceinline__ double whole_of(int chunks, F mass) {
    double v = 0.0;
    for (int c = threadIdx.x & 63; c < chunks; c += 64) v += mass(c);
    return wave_sum_d(v);
}

// The chunk in which the running share exceeds `want` (the last that has any, if none does) and the share before it; by
// every wave alike.  -1: no chunk has a share.
template <typename F>
__device__ __forceinline__ int chunk_at(int chunks, double want, double& at, F mass) {
    const int lane = threadIdx.x & 63;
    double before = 0.0;
    int ch = -1;
    for (int c0 = 0; c0 < chunks; c0 += 64) {
        const double m = c0 + lane < chunks ? mass(c0 + lane) : 0.0;
        const double run = before + wave_run_d(m);
        const uint64_t some = __ballot(m > 0.0), over = __ballot(m > 0.0 && run > want);
        const uint64_t take = over ? over & -over : some;
        if (take) {
            const int l = 63 - __clzll((long long)take);
            ch = c0 + l;
            at = __shfl(run - m, l);
        }
        if (over) break;
        before = __shfl(run, 63);
    }
    return __builtin_amdgcn_readfirstlane(ch);
}

// The token of chunk ch (of 64 * NV) in which the running share, `at` before the chunk, exceeds `want`, by the
// workgroup's first NV / EACH waves, EACH logits in a row a lane; every thread gets it.
template <bool DRAWN, int NV>
__device__ __forceinline__ int token_at(const mtp_verify_args& a, const Judged& j, int hide, int ch, double at, double want,
                                        double scale, RowLds& s) {
    constexpr int PW = NV / EACH;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (ch < 0) return -1;                       // uniform
    const int v0 = ch * 64 * NV + (int)threadIdx.x * EACH;
    double own[EACH], sum = 0.0;
    if (wave < PW) {
        // (the draft's row where one was refused: behind a row's last token there is none)
        const float *xp = a.logits + (int64_t)j.t * a.ld, *yp = DRAWN && j.refused ? a.draft + (int64_t)j.t * a.draft_ld : xp;
        float x[EACH], y[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int v = min(v0 + i, a.vocab - 1);
            x[i] = xp[v];
            if (DRAWN) y[i] = yp[v];
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int v = v0 + i;
            const float fx = shown(x[i], v, hide), fy = DRAWN ? shown(y[i], v, hide) : 0.f;
            own[i] = v < a.vocab ? share<DRAWN>(a, j, fx, fy, v, scale) : 0.0;
            sum += own[i];
        }
    }
    const double run = wave_run_d(wave < PW ? sum : 0.0);
    if (wave < PW && lane == 63) s.run[wave] = run;
    __syncthreads();
    if (wave < PW) {
        double x = at + (run - sum);
        for (int i = 0; i < wave; ++i) x += s.run[i];
        int first = 0x7fffffff, last = -1;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            x += own[i];
            if (own[i] > 0.0) {
                last = v0 + i;
                if (x > want) first = min(first, v0 + i);
            }
        }
        for (int o = 32; o; o >>= 1) {
            first = min(first, __shfl_xor(first, o));
            last = max(last, __shfl_xor(last, o));
        }
        if (lane == 0) { s.found[0][wave] = first; s.found[1][wave] = last; }
    }
    __syncthreads();
    int first = 0x7fffffff, last = -1;
    for (int i = 0; i < PW; ++i) {
        first = min(first, s.found[0][i]);
        last = max(last, s.found[1][i]);
    }
    return first != 0x7fffffff ? first : last;
}

// The shares of p in token t's chunks, of which c are the sums.
__device__ __forceinline__ double part_of(const Stat* c, int i, const Judged& j, double scale) {
    return c[i].sum * rel(c[i].max, j.pm, scale) * j.pz;
}

// What the drafts of row r came to, by a workgroup of nt threads: the accepted tokens, nothing behind them.
template <bool GREEDY>
__device__ __forceinline__ void emit(const mtp_verify_args& a, int r, const Row& row, const Judged& j, const RowLds& s, int nt) {
    for (int i = threadIdx.x; i < a.width; i += nt) {
        const bool in = i < j.live;
        a.token[(int64_t)r * a.width + i] = in ? s.draft[i] : -1;
        a.prob[(int64_t)r * a.width + i] = in ? (float)s.px[i] : 0.f;
    }
    if (threadIdx.x == 0) {
        a.count[r] = j.live;
        a.accepted[r] = j.accepted;
        a.done[r] = j.done;
    }
}
// The token drawn behind them, by one thread; hide: the id masked at its place.
template <bool GREEDY>
__device__ __forceinline__ void emit_drawn(const mtp_verify_args& a, int r, const Judged& j, int drawn, int hide, double scale) {
    if (drawn < 0) return;
    a.token[(int64_t)r * a.width + j.live] = drawn;
    a.prob[(int64_t)r * a.width + j.live] =
        GREEDY ? 1.f : (float)(rel(shown(a.logits[(int64_t)j.t * a.ld + drawn], drawn, hide), j.pm, scale) * j.pz);
    a.count[r] = j.live + 1;
    a.done[r] = drawn == a.eos_id ? 1 : 0;
}

// A row's draw and outputs by a workgroup of W waves that has judged it; stat: the row's chunks.  mass: room for the
// chunks' shares of max(p - q, 0), with DRAWN.
template <bool GREEDY, bool DRAWN, int NV, int W>
__device__ __forceinline__ void draw_row(const mtp_verify_args& a, int r, const Row& row, Judged j, const Stat* stat, int chunks,
                                         double scale, double* mass, RowLds& s) {
    emit<GREEDY>(a, r, row, j, s, 64 * W);
    if (j.i < 0) return;                         // uniform, as all that decides below
    const int hide = hidden(a, r, j.i), lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int drawn = j.at;
    if (!GREEDY) {
        const Stat* c = stat + (size_t)j.i * (DRAWN ? 2 : 1) * chunks;
        const double u = (double)a.uniforms[row.s];
        const int own = !DRAWN && j.refused && j.draft >= 0 && j.draft < a.vocab ? j.draft / (64 * NV) : -1;
        if (DRAWN && j.refused) {
            for (int i = wave; i < chunks; i += W) {
                const double m = chunk_mass<DRAWN, NV>(a, j, hide, i, scale);
                if (lane == 0) mass[i] = m;
            }
        } else if (own >= 0 && wave == 0) {
            const double m = chunk_mass<DRAWN, NV>(a, j, hide, own, scale);
            if (lane == 0) s.own = m;
        }
        __syncthreads();
        auto some = [&](int i) { return DRAWN && j.refused ? mass[i] : i == own ? s.own : part_of(c, i, j, scale); };
        auto all = [&](int i) { return part_of(c, i, j, scale); };
        double total = whole_of(chunks, some), at = 0.0;
        int ch;
        if (!(total > 0.0) && j.refused) {       // p is nowhere above q: from p itself
            j.refused = 0;
            total = whole_of(chunks, all);
            ch = chunk_at(chunks, u * total, at, all);
        } else {
            ch = chunk_at(chunks, u * total, at, some);
        }
        drawn = token_at<DRAWN, NV>(a, j, hide, ch, at, u * total, scale, s);
    }
    __syncthreads();                             // (the accepted ones' outputs come first)
    if (threadIdx.x == 0) emit_drawn<GREEDY>(a, r, j, drawn, hide, scale);
}

// One workgroup a row does everything: few chunks.
template <bool GREEDY, bool DRAWN>
__global__ __launch_bounds__(64 * NW) void verify_fused_kernel(mtp_verify_args a, double scale) {
    constexpr int NV = 8, PER = DRAWN ? 2 : 1;
    __shared__ RowLds s;
    __shared__ Stat s_stat[FUSED_UNITS];
    __shared__ double s_mass[FUSED_UNITS];
    const int r = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int chunks = chunks_of(a.vocab, NV);
    const Row row = row_of(a, r);
    const Draft mine = draft_of<GREEDY, DRAWN, NW>(a, row);
    for (int u = wave; u < row.n * PER * chunks; u += NW) {
        const int i = u / (PER * chunks), c = u - i * (PER * chunks), which = c / chunks, ch = c - which * chunks;
        if (which && i + 1 >= row.n) continue;
        const float* x = which ? a.draft + (int64_t)(row.s + i) * a.draft_ld : a.logits + (int64_t)(row.s + i) * a.ld;
        const Stat v = chunk_stat<GREEDY, NV>(x, a.vocab, ch, hidden(a, r, i), scale);
        if (lane == 0) s_stat[u] = v;
    }
    __syncthreads();
    const Judged j = judge<GREEDY, DRAWN, NW>(a, r, row, mine, s_stat, chunks, scale, s);
    draw_row<GREEDY, DRAWN, NV, NW>(a, r, row, j, s_stat, chunks, scale, s_mass, s);
}

// A wave a chunk of a token's logits (and draft logits).
template <bool GREEDY, bool DRAWN, int NV>
__global__ __launch_bounds__(256) void verify_chunk_kernel(mtp_verify_args a, VerifyWs w, int chunks, int groups, double scale) {
    constexpr int PER = DRAWN ? 2 : 1;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int u = blockIdx.x / groups, c = (blockIdx.x - u * groups) * 4 + wave;
    const int r = u / a.width, i = u - r * a.width;
    const Row row = row_of(a, r);
    const int which = c / chunks, ch = c - which * chunks;
    if (c >= PER * chunks || i + which >= row.n) return;
    const float* x = which ? a.draft + (int64_t)(row.s + i) * a.draft_ld : a.logits + (int64_t)(row.s + i) * a.ld;
    const Stat v = chunk_stat<GREEDY, NV>(x, a.vocab, ch, hidden(a, r, i), scale);
    if (lane == 0) w.stat[(size_t)u * PER * chunks + c] = v;
}

// A workgroup a row: drafts judged, and what p alone decides drawn.
template <bool GREEDY, int NV>
__global__ __launch_bounds__(64 * NW) void verify_row_kernel(mtp_verify_args a, VerifyWs w, int chunks, double scale) {
    __shared__ RowLds s;
    const int r = blockIdx.x;
    const Row row = row_of(a, r);
    const Stat* stat = w.stat + (size_t)r * a.width * chunks;
    const Judged j = judge<GREEDY, false, NW>(a, r, row, draft_of<GREEDY, false, NW>(a, row), stat, chunks, scale, s);
    draw_row<GREEDY, false, NV, NW>(a, r, row, j, stat, chunks, scale, nullptr, s);
}

// With draft logits: every workgroup of a row judges it, the first one writes what that gives, and each takes 16 chunks of
// 512 of max(p - q, 0) where a draft was refused.
__global__ __launch_bounds__(64 * NW) void verify_mass_kernel(mtp_verify_args a, VerifyWs w, int chunks, int parts, double scale) {
    __shared__ RowLds s;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = blockIdx.x / parts, c = (blockIdx.x - r * parts) * NW + wave, all = chunks_of(a.vocab, 8);
    const Row row = row_of(a, r);
    const Judged j = judge<false, true, NW>(a, r, row, draft_of<false, true, NW>(a, row), w.stat + (size_t)r * a.width * 2 * chunks, chunks, scale, s);
    if (blockIdx.x == r * parts) {
        emit<false>(a, r, row, j, s, 64 * NW);
        if (threadIdx.x == 0) w.judged[r] = j;
    }
    if (j.i < 0 || !j.refused || c >= all) return;
    const double m = chunk_mass<true, 8>(a, j, hidden(a, r, j.i), c, scale);
    if (lane == 0) w.mass[(size_t)r * all + c] = m;
}

template <int NV>
__global__ __launch_bounds__(256) void verify_pick_kernel(mtp_verify_args a, VerifyWs w, int chunks, double scale) {
    __shared__ RowLds s;
    const int r = blockIdx.x;
    const Row row = row_of(a, r);
    Judged j = w.judged[r];
    if (j.i < 0) return;
    const int parts = chunks_of(a.vocab, 8);
    const double* mass = w.mass + (size_t)r * parts;
    const Stat* c = w.stat + ((size_t)r * a.width + j.i) * 2 * chunks;
    const double u = (double)a.uniforms[row.s];
    const int hide = hidden(a, r, j.i);
    auto some = [&](int i) { return mass[i]; };
    auto all = [&](int i) { return part_of(c, i, j, scale); };
    double total = j.refused ? whole_of(parts, some) : 0.0, at = 0.0;
    int drawn;
    if (total > 0.0) {
        const int ch = chunk_at(parts, u * total, at, some);
        drawn = token_at<true, 8>(a, j, hide, ch, at, u * total, scale, s);
    } else {                                     // (nothing refused, or p nowhere above q)
        j.refused = 0;
        total = whole_of(chunks, all);
        const int ch = chunk_at(chunks, u * total, at, all);
        drawn = token_at<true, NV>(a, j, hide, ch, at, u * total, scale, s);
    }
    if (threadIdx.x == 0) emit_drawn<false>(a, r, j, drawn, hide, scale);
}

bool aligned(const void* p, uintptr_t n) { return p && ((uintptr_t)p & (n - 1)) == 0; }

// Logits a lane of a chunk: 8 where one workgroup a row does everything and where wider chunks would not fill the chip (2
// rows of 8 tokens over 32,000 logits, 512 chunks of 1024: 11.2 us with 8, 12.2 us with 16; 16 rows, 4096 chunks: 15.7 us
// either way; 32 rows of up to 8 over 65,536, the chunks alone: 23.0 us with 16, 26.5 us with 8, 24.0 us with 32).
int lane_logits(const mtp_verify_args& a) {
    return (int64_t)a.n_rows * a.width * chunks_of(a.vocab, WIDE_NV) * (a.draft ? 2 : 1) < 4096 ? 8 : WIDE_NV;
}
bool fused(const mtp_verify_args& a) {
    return (int64_t)a.width * chunks_of(a.vocab, 8) * (a.draft ? 2 : 1) <= FUSED_UNITS;
}

uint64_t carve(const mtp_verify_args& a, VerifyWs* w) {
    if (fused(a)) return 0;
    uint64_t o = 0;
    auto take = [&](uint64_t bytes) { uint64_t r = o; o = (o + bytes + 255) & ~uint64_t(255); return r; };
    const uint64_t chunks = chunks_of(a.vocab, lane_logits(a));
    const uint64_t s = take((uint64_t)a.n_rows * a.width * (a.draft ? 2 : 1) * chunks * sizeof(Stat));
    const uint64_t m = take(a.draft ? (uint64_t)a.n_rows * chunks_of(a.vocab, 8) * 8 : 0), j = take(a.draft ? a.n_rows * sizeof(Judged) : 0);
    if (w) {
        char* p = (char*)a.workspace;
        w->stat = (Stat*)(p + s); w->mass = (double*)(p + m); w->judged = (Judged*)(p + j);
    }
    return o;
}

int check(const mtp_verify_args* a) {
    if (!a) return MTP_EINVAL;
    if (a->n_rows < 0 || a->n_rows > 4096 || a->n_tokens < 0 || a->n_tokens >= (1 << 24) || a->vocab < 1 || a->vocab >= (1 << 24) ||
        a->width < 1 || a->width > MAX_WIDTH || a->eos_id < -1 || a->eos_id >= a->vocab || !(a->temperature >= 0.0) ||
        !isfinite(a->temperature) || (a->temperature > 0.0 && !isfinite(1.0 / a->temperature)))
        return MTP_EINVAL;
    // (a launch holds fewer than 2^24 workgroups of 256 threads, 2^22 of 1024; chunks of 512 are taken where there are few)
    if ((int64_t)a->n_rows * a->width * ((chunks_of(a->vocab, WIDE_NV) * 2 + 3) / 4) >= (1ll << 24)) return MTP_EINVAL;
    if ((int64_t)a->n_rows * ((chunks_of(a->vocab, 8) + NW - 1) / NW) >= (1ll << 22)) return MTP_EINVAL;
    return MTP_OK;
}

template <bool GREEDY, bool DRAWN, int NV>
void wide_go(hipStream_t st, const mtp_verify_args& a, const VerifyWs& w, double scale) {
    const int chunks = chunks_of(a.vocab, NV), groups = (chunks * (DRAWN ? 2 : 1) + 3) / 4, parts = (chunks_of(a.vocab, 8) + NW - 1) / NW;
    hipLaunchKernelGGL((verify_chunk_kernel<GREEDY, DRAWN, NV>), dim3((unsigned)(a.n_rows * a.width * groups)), dim3(256), 0, st, a, w,
                       chunks, groups, scale);
    if constexpr (DRAWN) {
        hipLaunchKernelGGL(verify_mass_kernel, dim3((unsigned)(a.n_rows * parts)), dim3(64 * NW), 0, st, a, w, chunks, parts, scale);
        hipLaunchKernelGGL(verify_pick_kernel<NV>, dim3(a.n_rows), dim3(256), 0, st, a, w, chunks, scale);
    } else {
        hipLaunchKernelGGL((verify_row_kernel<GREEDY, NV>), dim3(a.n_rows), dim3(64 * NW), 0, st, a, w, chunks, scale);
    }
}

template <bool GREEDY, bool DRAWN>
int go(hipStream_t st, const mtp_verify_args& a, const VerifyWs& w, int nv) {
    // (finite, so that 0 times it is 0)
    const double scale = GREEDY ? 0.0 : std::min(1.4426950408889634074 / a.temperature, std::numeric_limits<double>::max());
    if (fused(a)) hipLaunchKernelGGL((verify_fused_kernel<GREEDY, DRAWN>), dim3(a.n_rows), dim3(64 * NW), 0, st, a, scale);
    else if (nv == 8) wide_go<GREEDY, DRAWN, 8>(st, a, w, scale);
    else wide_go<GREEDY, DRAWN, WIDE_NV>(st, a, w, scale);
    return hipGetLastError() == hipSuccess ? MTP_OK : MTP_EHIP;
}

}  // namespace
}  // namespace mtp

extern "C" {

int mtp_verify_drafts_workspace_size(const mtp_verify_args* args, uint64_t* bytes) {
    if (mtp::check(args) != MTP_OK || !bytes) return MTP_EINVAL;
    *bytes = mtp::carve(*args, nullptr);
    return MTP_OK;
}

int mtp_verify_drafts(const mtp_verify_args* args, void* hip_stream) {
    using namespace mtp;
    const int rc = check(args);
    if (rc != MTP_OK) return rc;
    const mtp_verify_args& a = *args;
    if (a.n_rows == 0) return MTP_OK;
    if (!aligned(a.row_start, 4) || !aligned(a.token, 4) || !aligned(a.prob, 4) || !aligned(a.count, 4) || !aligned(a.accepted, 4) ||
        !aligned(a.done, 4) || (a.eos_id >= 0 && a.eos_min > 0 && !aligned(a.len, 4)))
        return MTP_EINVAL;
    if (a.n_tokens > 0 && (!aligned(a.logits, 4) || a.ld < a.vocab || !aligned(a.tokens, 4) || !aligned(a.uniforms, 4) ||
                           (a.draft && (!aligned(a.draft, 4) || a.draft_ld < a.vocab))))
        return MTP_EINVAL;
    VerifyWs w{};
    const uint64_t need = carve(a, &w);
    if (need && !aligned(a.workspace, 256)) return MTP_EINVAL;
    if (need > a.workspace_bytes) return MTP_ENOMEM;
    hipStream_t st = (hipStream_t)hip_stream;
    // (with temperature 0 the draft's distribution changes nothing)
    if (a.temperature == 0.0) {
        mtp_verify_args g = a;
        g.draft = nullptr;
        return go<true, false>(st, g, w, lane_logits(a));
    }
    return a.draft ? go<false, true>(st, a, w, lane_logits(a)) : go<false, false>(st, a, w, lane_logits(a));
}

}  // extern "C"
