// Attention over a paged cache that adds up the weight each cached token got
// (mtp_pages_attention_weights).  See include/mtp.h for the operator's definition.
//
//   w[row][KV head][j] += sum over the row's queries t and the head's query heads h of p_thj,
//   p_thj = exp2(s_thj - m_th) f_th
//
// The attention leaves every query's reference m and factor f.  With few queries it
// stores their scores too and sums their probabilities itself, key by key; with many it
// would cost more to store the scores than to form them again, here: S^T[key][q] =
// K[key][:] . Q[q][:], a wave's 32 keys held in registers while the row's queries
// pass, and every lane sums its queries' probabilities of its own keys.  A key belongs
// to one wave (or thread) and the queries come in order, so that the sums do not depend
// on scheduling.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "../../include/mtp.h"
#include "common.h"
#include "page_attn.h"
#include "wave.h"

namespace mtp {
namespace {

constexpr int PG = 16;
constexpr float LOG2E = 1.4426950408889634f;
constexpr int NW = 4;
constexpr int WK = 32;                           // keys of a wave
constexpr int BK = NW * WK;                      // keys of a workgroup's block

struct WeighArgs {
    mtp_attention_args a;
    const float2* ref;
    float* weights;
    int64_t ld;
    int runs;                                    // workgroups per row and head
};

// 32 keys in operand order, as the attention over few query rows has them: bf16, row 4 g + e of tile t is key 8 g + 4 t +
// e, so that lane (q, g) ends with the scores of keys 8 g .. + 7; fp32, of keys 16 t + 4 g + e.
template <typename T, int D>
struct Operand {
    uint4 k[2][D * sizeof(T) / 64];
    __device__ __forceinline__ void load(const T* p0, const T* p1, int r, int g) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const T* p = sizeof(T) == 2 ? (r & 8 ? p1 : p0) + (8 * ((r >> 2) & 1) + (r & 3) + 4 * t) * D + 8 * g
                                        : (t ? p1 : p0) + r * D + 4 * g;
#pragma unroll
            for (int j = 0; j < D * (int)sizeof(T) / 64; ++j) k[t][j] = *reinterpret_cast<const uint4*>(p + (sizeof(T) == 2 ? 32 : 16) * j);
        }
    }
};

template <typename T, int D>
__global__ __launch_bounds__(64 * NW) void weigh_kernel(WeighArgs w) {
    const mtp_attention_args& a = w.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, gr = lane >> 4;
    const int H = a.cache.n_kv_heads, G = a.n_heads / H;
    const int hk = blockIdx.x % H, u = blockIdx.x / H, c = u / w.runs, run = u - c * w.runs;
    const int s = max(0, min(a.row_start[c], a.n_tokens)), n = max(0, min(a.row_start[c + 1], a.n_tokens) - s);
    const int kv = max(0, min(a.kv_len[c], PG * a.max_pages));
    if (n == 0) return;
    const bool causal = a.mode == MTP_ATTN_CAUSAL;
    const int64_t first = (int64_t)kv - n;                               // the first query's position
    const size_t vofs = (size_t)H * PG * D, pstr = 2 * vofs;
    const T* pool = (const T*)a.cache.pool + (size_t)hk * PG * D;
    const int32_t* tab = a.table + (size_t)c * a.max_pages;
    float* out = w.weights + ((size_t)c * H + hk) * w.ld;
    const float scale = a.scale * LOG2E;

    for (int b = run; (int64_t)b * BK < kv; b += w.runs) {
        const int kb = b * BK + wave * WK;
        if (kb >= kv) return;
        if (causal && a.window > 0 && kb + WK <= first - a.window + 1) continue;                  // before every window
        int x0 = tab[kb / PG], x1 = kb + PG < kv ? tab[kb / PG + 1] : -1;
        x0 = x0 >= 0 && x0 < a.cache.num_pages ? x0 : -1;
        x1 = x1 >= 0 && x1 < a.cache.num_pages ? x1 : -1;
        Operand<T, D> k;
        k.load(pool + (size_t)max(x0, 0) * pstr, pool + (size_t)max(x1, 0) * pstr, r, gr);
        if (a.scale == 0.f) {                    // scores are 0, also where the product would be infinite
#pragma unroll
            for (int j = 0; j < D * (int)sizeof(T) / 64; ++j) k.k[0][j] = k.k[1][j] = make_uint4(0, 0, 0, 0);
        }
        auto key_of = [&](int u) { return kb + (sizeof(T) == 2 ? 8 * gr + u : 16 * (u >> 2) + 4 * gr + (u & 3)); };
        auto there = [&](int u) { return (key_of(u) - kb < PG ? x0 : x1) >= 0 && key_of(u) < kv; };
        // the row's queries that see any of these keys: [i0, i1)
        int i0 = 0, i1 = n;
        if (causal) {
            i0 = (int)max((int64_t)0, kb - first);
            if (a.window > 0) i1 = (int)max((int64_t)0, min((int64_t)n, kb + WK - 1 + (int64_t)a.window - first));
        }
        float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int64_t q0 = (int64_t)i0 * G; q0 < (int64_t)i1 * G; q0 += 16) {
            const int64_t row = min(q0 + r, (int64_t)i1 * G - 1);
            const int i = (int)((uint32_t)row / (uint32_t)G), h = (int)(row - (int64_t)i * G);
            const T* qp = (const T*)a.q + (int64_t)(s + i) * a.q_stride + (hk * G + h) * D;
            float2 ref = w.ref[(int64_t)(s + i) * a.n_heads + hk * G + h];
            if (q0 + r > row) ref.y = 0.f;                               // behind the last
            uint4 q[D * sizeof(T) / 64];
#pragma unroll
            for (int j = 0; j < D * (int)sizeof(T) / 64; ++j)
                q[j] = *reinterpret_cast<const uint4*>(qp + (sizeof(T) == 2 ? 32 * j + 8 * gr : 16 * j + 4 * gr));
            const int64_t pos = first + i, lo = causal ? (a.window > 0 ? pos - a.window + 1 : 0) : 0, hi = causal ? pos + 1 : kv;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x4_t sc = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < D * (int)sizeof(T) / 64; ++j) {
                    if constexpr (sizeof(T) == 2) {
                        sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k.k[t][j]),
                                                                     __builtin_bit_cast(bf16x8_t, q[j]), sc, 0, 0, 0);
                    } else {
                        const float4 kk = __builtin_bit_cast(float4, k.k[t][j]), qq = __builtin_bit_cast(float4, q[j]);
                        sc = __builtin_amdgcn_mfma_f32_16x16x4f32(kk.x, qq.x, sc, 0, 0, 0);
                        sc = __builtin_amdgcn_mfma_f32_16x16x4f32(kk.y, qq.y, sc, 0, 0, 0);
                        sc = __builtin_amdgcn_mfma_f32_16x16x4f32(kk.z, qq.z, sc, 0, 0, 0);
                        sc = __builtin_amdgcn_mfma_f32_16x16x4f32(kk.w, qq.w, sc, 0, 0, 0);
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
#pragma clang fp contract(off)                   // (the attention rounds the scaled score, too)
                    const int u = 4 * t + e, key = key_of(u);
                    const bool in = ref.y > 0.f && key >= lo && key < hi && there(u);
                    const float p = __builtin_amdgcn_exp2f(sc[e] * scale - ref.x) * ref.y;
                    acc[u] += in ? p : 0.f;
                }
            }
        }
        // the sums over a key's 16 lanes; lane u < 8 of them writes key u
        float mine = 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float v = sum16(acc[u]);
            mine = r == u ? v : mine;
        }
        const int key = key_of(r & 7);
        if (r < 8 && key < kv) out[key] = (causal && key >= first ? 0.f : out[key]) + mine;
    }
}

// ------------------------------------------------------------ many query rows
//
// bf16: 32 x 32 x 16 products.  A workgroup's four waves take 32 keys each; 64 query
// rows at a time come through LDS, the next ones' loads going straight there while the
// current ones are used.  Lane (q, h) of a 32 x 32 tile has query q's scores of keys 8
// (i / 4) + 4 h + i % 4.  A row's 16-byte pieces are stored in an order that the row
// shifts (by the address that a lane loads from), so that 16 lanes read different banks.
// What bounds it: the vector unit (an exponential and two fused products a score, 96 of
// the 113 instructions' cycles that a 32 x 32 tile takes; busy 55% of the time, the matrix
// cores 27%) and waits at the barriers that three workgroups a CU do not hide.  Chunks of
// 400 to 512 tokens over 2048 to 8192 keys, 32 query heads on 8 KV heads of 128: 117 to 132
// us (two workgroups a CU 140 to 150 us, four of 128 registers, one 32 x 32 product at a
// time, 137 us; rows found by a division each step 140 us; the keys' first wait inside the
// loop, where it is one for the queries under way too, 130 us).
constexpr int QR = 64;                           // query rows of a step

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef const __attribute__((address_space(1))) void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

template <int D>
__global__ __launch_bounds__(64 * NW, 3) void weigh_tile_kernel(WeighArgs w) {
    constexpr int CW = D / 8;                    // pieces of a row
    __shared__ __attribute__((aligned(1024))) bf16_t s_q[2][QR * D];
    __shared__ float s_m[2][QR], s_f[2][QR];     // references and factors
    __shared__ int s_tok[2][QR];                 // tokens of the row
    static_assert(QR == 64, "a lane a row");
    const mtp_attention_args& a = w.a;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int qc = lane & 31, hh = lane >> 5;
    const int H = a.cache.n_kv_heads, G = a.n_heads / H;
    const int hk = blockIdx.x % H, u = blockIdx.x / H, c = u / w.runs, run = u - c * w.runs;
    const int s = max(0, min(a.row_start[c], a.n_tokens)), n = max(0, min(a.row_start[c + 1], a.n_tokens) - s);
    const int kv = max(0, min(a.kv_len[c], PG * a.max_pages));
    if (n == 0) return;
    const bool causal = a.mode == MTP_ATTN_CAUSAL;
    const int64_t first = (int64_t)kv - n;
    const size_t vofs = (size_t)H * PG * D, pstr = 2 * vofs;
    const bf16_t* pool = (const bf16_t*)a.cache.pool + (size_t)hk * PG * D;
    const int32_t* tab = a.table + (size_t)c * a.max_pages;
    float* out = w.weights + ((size_t)c * H + hk) * w.ld;
    const float scale = fabsf(a.scale) * LOG2E;
    const int qsw = D == 128 ? qc & 15 : (qc >> 1) & 7;

    for (int b = run; (int64_t)b * BK < kv; b += w.runs) {
        if (causal && a.window > 0 && ((int64_t)b + 1) * BK <= first - a.window + 1) continue;    // before every window
        const int kb = b * BK + wave * WK;
        auto page_of = [&](int key) {
            const int x = key < kv ? tab[key / PG] : -1;
            return x >= 0 && x < a.cache.num_pages ? x : -1;
        };
        const int x0 = page_of(kb), x1 = page_of(kb + PG);
        bf16x8_t k[D / 16];
        const bf16_t* kp = pool + (size_t)max(qc < PG ? x0 : x1, 0) * pstr + (qc % PG) * D + 8 * hh;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) k[j] = *reinterpret_cast<const bf16x8_t*>(kp + 16 * j);
        // (scores as the attention over many query rows forms them, times a scale above 0; of scale 0 they are 0, also where
        // the product would be infinite)
        if (a.scale <= 0.f) {
            typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                const u32x4_t v = __builtin_bit_cast(u32x4_t, k[j]);
                k[j] = __builtin_bit_cast(bf16x8_t, a.scale == 0.f ? u32x4_t{0, 0, 0, 0} : v ^ 0x80008000u);
            }
        }
        // the row's queries that see any key of the block: [i0, i1)
        int64_t i0 = 0, i1 = n;
        if (causal) {
            i0 = max((int64_t)0, (int64_t)b * BK - first);
            if (a.window > 0) i1 = max((int64_t)0, min((int64_t)n, (int64_t)b * BK + BK - 1 + a.window - first));
        }
        const int r0 = (int)min(i0 * G, (int64_t)n * G), r1 = (int)max((int64_t)r0, i1 * G);
        // A lane's rows of a step, as token, head and address: they go on by 64 rows a step (a division by the group and a
        // product for each cost more than the matrix products).  Behind the last row the last one stands in.
        const int di = QR / G, dh = QR % G, end = (int)i1;
        const int64_t step = (int64_t)di * a.q_stride + dh * D, wrap = a.q_stride - (int64_t)G * D;
        const bf16_t* const q_at = (const bf16_t*)a.q + (int64_t)s * a.q_stride + (int64_t)hk * G * D;
        struct Row { int i, h; const bf16_t* p; };
        auto row_at = [&](int q, int piece) { return Row{q / G, q % G, q_at + (int64_t)(q / G) * a.q_stride + (q % G) * D + piece * 8}; };
        auto next = [&](Row& x) {
            const bool over = x.h + dh >= G;
            x.p += step + (over ? wrap : 0);
            x.i += over ? di + 1 : di;
            x.h += over ? dh - G : dh;
        };
        constexpr int FLY = QR * CW / 256;
        Row at[FLY], own = row_at(r0 + lane, 0);
        const bf16_t* last[FLY];                 // (a row's pieces in the order that its place in the step shifts)
#pragma unroll
        for (int f = 0; f < FLY; ++f) {
            const int in = f * 256 + tid, row = in / CW, piece = (in % CW) ^ (D == 128 ? row & 15 : (row >> 1) & 7);
            at[f] = row_at(r0 + row, piece);
            last[f] = q_at + (int64_t)(end - 1) * a.q_stride + (G - 1) * D + piece * 8;
        }
        auto stage = [&](int buf) {
#pragma unroll
            for (int f = 0; f < FLY; ++f) {
                const bf16_t* src = at[f].i < end ? at[f].p : last[f];
                __builtin_amdgcn_global_load_lds((gptr_t)src, (lptr_t)(&s_q[buf][(f * 256 + wave * 64) * 8]), 16, 0, 0);
                next(at[f]);
            }
            if (wave == 0) {
                const bool out = own.i >= end;
                const float* ref = (const float*)(w.ref + (int64_t)(s + (out ? end - 1 : own.i)) * a.n_heads + hk * G + (out ? G - 1 : own.h));
                __builtin_amdgcn_global_load_lds((gptr_t)ref, (lptr_t)(&s_m[buf][0]), 4, 0, 0);
                __builtin_amdgcn_global_load_lds((gptr_t)(ref + 1), (lptr_t)(&s_f[buf][0]), 4, 0, 0);
                s_tok[buf][lane] = own.i;
                next(own);
            }
        };
        float acc[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = 0.f;
        const bool all_there = x0 >= 0 && x1 >= 0 && kb + WK <= kv;
        // (the keys' loads end before the loop, where a wait for them would be one for the queries on their way too)
        __builtin_amdgcn_s_waitcnt(0x0f70);      // vmcnt(0)
        if (r0 < r1) stage(0);
        // query rows [w0, w1) see all of the wave's keys
        int w0 = r1, w1 = r0;
        if (all_there) {
            auto rows_of = [&](int64_t t) { return (int)max((int64_t)r0, min((int64_t)r1, t * G)); };
            w0 = causal ? rows_of(kb + WK - 1 - first) : r0;
            w1 = causal && a.window > 0 ? rows_of(kb + (int64_t)a.window - first) : r1;
        }
        int q0 = r0, buf = 0;
        // this wave's loads of the step have landed; all waves' have, and all are done with the other buffer
        auto arrive = [&]() {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if (q0 + QR < r1) stage(buf ^ 1);
        };
        f32x16_t sc[QR / 32];
        float m[QR / 32], f[QR / 32];
        auto scores = [&]() {
#pragma unroll
            for (int t = 0; t < QR / 32; ++t) {
                m[t] = s_m[buf][32 * t + qc];
                f[t] = s_f[buf][32 * t + qc];
                const bf16_t* q = &s_q[buf][(32 * t + qc) * D];
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[t][i] = 0.f;
#pragma unroll
                for (int j = 0; j < D / 16; ++j)
                    sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        k[j], *reinterpret_cast<const bf16x8_t*>(q + ((2 * j + hh) ^ qsw) * 8), sc[t], 0, 0, 0);
            }
        };
        while (q0 < r1) {
            // (a loop of its own: in one with the masks the sums were copied every step)
            for (; q0 >= w0 && q0 + QR <= w1; q0 += QR, buf ^= 1) {
                arrive();
                scores();
#pragma unroll
                for (int t = 0; t < QR / 32; ++t) {
                    if (__any(!(f[t] > 0.f))) {  // queries that add nothing, whose scores may be anything
#pragma unroll
                        for (int i = 0; i < 16; ++i) sc[t][i] = f[t] > 0.f ? sc[t][i] : 0.f;
                    }
                    m[t] = f[t] > 0.f ? m[t] : 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[i] = fmaf(__builtin_amdgcn_exp2f(fmaf(sc[t][i], scale, -m[t])), f[t], acc[i]);
                }
            }
            if (q0 >= r1) break;
            arrive();
            scores();
#pragma unroll
            for (int t = 0; t < QR / 32; ++t) {
                const int tok = s_tok[buf][32 * t + qc];
                const int64_t pos = first + tok, lo = causal && a.window > 0 ? pos - a.window + 1 : 0;
                const int64_t hi = causal ? min((int64_t)kv, pos + 1) : kv;
                // keys [k0, k1) of the wave's 32, none for a query that adds nothing
                const int k0 = (int)max((int64_t)0, min((int64_t)WK, lo - kb));
                const int k1 = tok < end && f[t] > 0.f ? (int)max((int64_t)0, min((int64_t)WK, hi - kb)) : 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int in = 8 * (i >> 2) + 4 * hh + (i & 3);
                    const float p = __builtin_amdgcn_exp2f(fmaf(sc[t][i], scale, -m[t])) * f[t];
                    acc[i] += in >= k0 && in < k1 && (i < 8 ? x0 : x1) >= 0 ? p : 0.f;
                }
            }
            q0 += QR;
            buf ^= 1;
        }
        // the sums over a key's 32 lanes; lane (i, h) writes the key of register i
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float v = xor16_sum(sum16(acc[i]));
            sum = qc == i ? v : sum;
        }
        const int key = kb + 8 * (qc >> 2) + 4 * hh + (qc & 3);
        if (qc < 16 && key < kv) out[key] = (causal && key >= first ? 0.f : out[key]) + sum;
        __syncthreads();                         // (the next block's queries overwrite this one's)
    }
}

bool aligned(const void* p, uintptr_t n) { return p && ((uintptr_t)p & (n - 1)) == 0; }

int check(const mtp_weigh_args* a) {
    if (!a) return MTP_EINVAL;
    const int rc = attention_check(&a->attention);
    if (rc != MTP_OK) return rc;
    return a->ld < (int64_t)PG * a->attention.max_pages ? MTP_EINVAL : MTP_OK;
}

// What a call does: scores stored or formed again (by which kernel), and its workspace: the attention's own, the queries'
// references, the scores.
struct WeighCut {
    bool stored, tiles;
    uint64_t ref_at, score_at, bytes;
};

// Stored where a key has 16 times as many bytes as it has queries, and no more than 256 MB of scores in all (16 single
// tokens over 4000 keys, four query heads on each of 8 KV heads of 128 in bf16, 64 bytes a query: 53 us stored, 79 us formed
// again; at the border, 16 bytes, neither is 5% ahead: fp32, head dim 128, 32 queries 96 and 98 us, bf16, head dim 64, 8
// queries 24.4 and 23.3 us; past it, bf16, head dim 64, 16 queries 27.5 and 23.9 us).  Their room is that of the table,
// since max_kv is a hint that a row may exceed: a table far wider than its rows forms them again (32 single tokens over 500
// to 2000 keys, 32 heads on 8 of 128: 41 us with tables of 125 or 1024 pages, 53 us with 8192, max_kv 2000; 4 tokens a row
// 65 and 64 us).  Else 32 x 32 tiles for bf16 rows of 64 queries and more on average (16 rows over 2000 keys
// of 8 heads of 128: 64 queries 59 us in tiles of 32 and 66 us in tiles of 16, 32 queries 64 and 61 us; of 4 heads of 64:
// 64 queries 31.5 us either way, 32 queries 29.0 and 25.8 us).
WeighCut weigh_cut(const mtp_attention_args& a) {
    WeighCut x{};
    const int64_t group = a.n_heads / a.cache.n_kv_heads, cap = (int64_t)PG * a.max_pages;
    const int64_t rows = a.n_tokens * group, key = a.cache.head_dim * (a.cache.dtype == MTP_DTYPE_BF16 ? 2 : 4);
    const int64_t scores = (int64_t)a.n_tokens * a.n_heads * cap * 4;
    x.stored = !attention_wide(a) && 16 * rows <= key * a.n_rows && scores <= (1ll << 28);
    x.tiles = a.cache.dtype == MTP_DTYPE_BF16 && rows >= 64ll * a.n_rows;
    auto up = [](uint64_t n) { return (n + 255) & ~uint64_t(255); };
    x.ref_at = up(attention_bytes(a));
    x.score_at = up(x.ref_at + (uint64_t)a.n_tokens * a.n_heads * 8);
    x.bytes = x.stored ? x.score_at + scores : x.score_at;
    return x;
}

// Workgroups per row and KV head for blocks of `keys`: 8192 in all at most, where there are more a workgroup takes several.
int runs_of(const mtp_attention_args& a, int keys) {
    int64_t kv = (int64_t)PG * a.max_pages;
    if (a.max_kv > 0) kv = std::min<int64_t>(kv, a.max_kv);
    const int64_t work = (int64_t)a.n_rows * a.cache.n_kv_heads;
    return (int)std::max<int64_t>(1, std::min<int64_t>((kv + keys - 1) / keys, (8192 + work - 1) / work));
}

int weigh_go(hipStream_t st, WeighArgs& w, const WeighCut& x) {
    const mtp_attention_args& a = w.a;
    w.runs = runs_of(a, BK);
    const dim3 grid((unsigned)(a.n_rows * a.cache.n_kv_heads * w.runs)), threads(64 * NW);
    const bool bf = a.cache.dtype == MTP_DTYPE_BF16, d64 = a.cache.head_dim == 64;
    if (x.tiles && d64) hipLaunchKernelGGL(weigh_tile_kernel<64>, grid, threads, 0, st, w);
    else if (x.tiles) hipLaunchKernelGGL(weigh_tile_kernel<128>, grid, threads, 0, st, w);
    else if (bf && d64) hipLaunchKernelGGL((weigh_kernel<bf16_t, 64>), grid, threads, 0, st, w);
    else if (bf) hipLaunchKernelGGL((weigh_kernel<bf16_t, 128>), grid, threads, 0, st, w);
    else if (d64) hipLaunchKernelGGL((weigh_kernel<float, 64>), grid, threads, 0, st, w);
    else hipLaunchKernelGGL((weigh_kernel<float, 128>), grid, threads, 0, st, w);
    return hipGetLastError() == hipSuccess ? MTP_OK : MTP_EHIP;
}

}  // namespace
}  // namespace mtp

extern "C" {

int mtp_pages_attention_weights_workspace_size(const mtp_weigh_args* args, uint64_t* bytes) {
    using namespace mtp;
    if (check(args) != MTP_OK || !bytes) return MTP_EINVAL;
    const mtp_attention_args& a = args->attention;
    *bytes = a.n_rows == 0 || a.n_tokens == 0 ? 0 : weigh_cut(a).bytes;
    return MTP_OK;
}

int mtp_pages_attention_weights(const mtp_weigh_args* args, void* hip_stream) {
    using namespace mtp;
    int rc = check(args);
    if (rc != MTP_OK) return rc;
    WeighArgs w{args->attention, nullptr, args->weights, args->ld, 0};
    mtp_attention_args& a = w.a;
    if (a.n_rows == 0 || a.n_tokens == 0) return MTP_OK;
    if (!aligned(w.weights, 4) || !aligned(a.workspace, 256)) return MTP_EINVAL;
    const WeighCut x = weigh_cut(a);
    if (a.workspace_bytes < x.bytes) return MTP_ENOMEM;
    float2* ref = (float2*)((char*)a.workspace + x.ref_at);
    float* score = x.stored ? (float*)((char*)a.workspace + x.score_at) : nullptr;
    hipStream_t st = (hipStream_t)hip_stream;
    rc = attention_run(a, ref, score, AttnSums{w.weights, w.ld}, st);
    if (rc != MTP_OK || x.stored) return rc;
    w.ref = ref;
    return weigh_go(st, w, x);
}

}  // extern "C"
