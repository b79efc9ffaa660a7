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

#include <algorithm>

#include "../../include/mtp.h"
#include "common.h"
#include "wave.h"

namespace mtp {

int cache_check(const mtp_cache& c);

namespace {

constexpr int PG = 16;
constexpr float LOG2E = 1.4426950408889634f;
constexpr int MAX_RUNS = 256;                    // of a tile's keys

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

// How a call is cut.  A tile is up to tt tokens of one row times the gs query
// heads of one block (hb blocks make the group of a KV head): query row r of a
// tile is token r / gs, head r % gs, so that grouped heads share the keys they
// load.  Tiles are numbered row by row: row c owns the numbers row_start[c] /
// tt + c up to the next row's first (at least as many as it needs; the others
// are empty), so a workgroup finds its row by a search and the host needs no
// lengths.  The keys of a tile are cut into n_splits runs of split_len, the
// last one taking whatever is behind them; a tile with more than one live run
// leaves partial sums for a second launch.
struct AttnGeo {
    int gs, hb, tt, n_tiles, n_splits, split_len;
    int sorted;                // workgroups in the order of find_item
    float* acc;                // [n_tiles * heads * hb][n_splits][tile rows][D]
    float2* ml;                // [...][tile rows] reference and sum
};

struct AttnTile {
    int c, t0, nt;             // cache row, first token, tokens (0: empty)
    int kv, pos0;              // the row's keys, the first token's position
    int lo, hi;                // positions that some query of the tile sees
};

__device__ __forceinline__ int start_of(const mtp_attention_args& a, int c) {
    return max(0, min(a.row_start[c], a.n_tokens));
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Tile `local` of row c, whose tokens are [s, e).
__device__ __forceinline__ AttnTile tile_at(const mtp_attention_args& a, const AttnGeo& g, int c, int s, int e, int kv,
                                            int local) {
    AttnTile t;
    t.c = c;
    t.t0 = s + local * g.tt;
    t.nt = local < 0 ? 0 : max(0, min(g.tt, e - t.t0));
    t.kv = kv;
    t.pos0 = t.kv - (e - s) + (t.t0 - s);
    t.lo = 0;
    t.hi = t.kv;
    if (a.mode == MTP_ATTN_CAUSAL) {
        t.hi = max(0, min(t.kv, t.pos0 + t.nt));
        if (a.window > 0) t.lo = max(0, t.pos0 - a.window + 1);
    }
    return t;
}
__device__ __forceinline__ int keys_of(const mtp_attention_args& a, int c) {
    return max(0, min(a.kv_len[c], PG * a.max_pages));
}

// The tile's row, found by the whole wave, 64 candidates a round; uniform.
__device__ __forceinline__ AttnTile find_tile(const mtp_attention_args& a, const AttnGeo& g, int tile) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = a.n_rows;                    // the row lies in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 63) >> 6, i = lane * step;
        const bool le = i < n && start_of(a, lo + min(i, n - 1)) / g.tt + lo + i <= tile;
        const int k = max(1, (int)__popcll(__ballot(le)));
        lo += (k - 1) * step;
        n = min(step, n - (k - 1) * step);
    }
    const int c = __builtin_amdgcn_readfirstlane(lo);
    const int s = start_of(a, c), e = start_of(a, c + 1);
    return tile_at(a, g, c, s, e, keys_of(a, c), tile - (s / g.tt + c));
}

// Work item u of a head: a tile and a run of its keys; the whole runs of every
// row first, then the rows' rests, the longest first, and nothing (no tokens)
// behind them: workgroups start in this order, so that the last ones to start
// are short.  A lane each row; unsorted, tiles in order, run by run.
__device__ __forceinline__ AttnTile find_item(const mtp_attention_args& a, const AttnGeo& g, int u, int& tile, int& split) {
    if (!g.sorted) {
        split = uniform(u / g.n_tiles);
        tile = u - split * g.n_tiles;
        return find_tile(a, g, tile);
    }
    const int lane = threadIdx.x & 63, c = min(lane, a.n_rows - 1);
    const int s = start_of(a, c), e = start_of(a, c + 1), kv = keys_of(a, c);
    const int count = lane < a.n_rows && e > s ? (e - s + g.tt - 1) / g.tt : 0;
    // what a tile sees of them (in a window from a multiple of 32 on, as runs_of cuts it)
    const int see = a.window > 0 ? min(kv, a.window + g.tt + 31) : kv;
    const int whole = min(see / g.split_len, g.n_splits), rest = whole < g.n_splits ? see - whole * g.split_len : -1;
    const int c0 = count * whole, c1 = rest >= 0 ? count : 0;
    int b0 = 0, b1 = 0, all0 = 0;                // items before this lane's whole runs and before its rest
    for (int k = 0; k < a.n_rows; ++k) {
        const int k0 = __builtin_amdgcn_readlane(c0, k), k1 = __builtin_amdgcn_readlane(c1, k);
        const int kr = __builtin_amdgcn_readlane(rest, k);
        all0 += k0;
        b0 += k < lane ? k0 : 0;
        b1 += kr > rest || (kr == rest && k < lane) ? k1 : 0;
    }
    const bool first = u < all0;
    const int at = first ? u - b0 : u - all0 - b1, n = first ? c0 : c1;
    const uint64_t hit = __ballot(at >= 0 && at < n);
    const int l = hit ? __ffsll((unsigned long long)hit) - 1 : 0;
    const int rs = __builtin_amdgcn_readlane(s, l), rc = max(1, __builtin_amdgcn_readlane(count, l));
    const int i = __builtin_amdgcn_readlane(at, l), run = first ? i / rc : __builtin_amdgcn_readlane(whole, l);
    const int local = first ? i - run * rc : i;
    split = uniform(run);
    tile = uniform(rs / g.tt + l + local);
    return tile_at(a, g, uniform(l), rs, __builtin_amdgcn_readlane(e, l), __builtin_amdgcn_readlane(kv, l),
                   uniform(hit ? local : -1));
}

// The keys [k0, k1) of run `split`, and the number of live runs (at least 1;
// a tile that sees nothing has one empty run).
__device__ __forceinline__ int runs_of(const AttnGeo& g, const AttnTile& t, int split, int& k0, int& k1) {
    const int base = t.lo & ~31;
    const int live = min(g.n_splits, max(1, (t.hi - base + g.split_len - 1) / g.split_len));
    k0 = base + split * g.split_len;
    k1 = split == live - 1 ? t.hi : min(t.hi, k0 + g.split_len);
    return live;
}

// What query row r of the tile sees: [lo, hi).
__device__ __forceinline__ void sight_of(const mtp_attention_args& a, const AttnGeo& g, const AttnTile& t, int r, int& lo,
                                         int& hi) {
    lo = 0;
    hi = t.kv;
    if (a.mode == MTP_ATTN_CAUSAL) {
        const int pos = t.pos0 + r / g.gs;
        hi = min(t.kv, pos + 1);
        if (a.window > 0) lo = max(0, pos - a.window + 1);
    }
}

__device__ __forceinline__ uint32_t pk2(float a, float b) { return bf16x2_bits(a, b); }

// Two bf16 with those that are not finite set to zero.
__device__ __forceinline__ uint32_t finite2(uint32_t v) {
    const bool lo = (v & 0x7f80u) == 0x7f80u, hi = (v & 0x7f800000u) == 0x7f800000u;
    return v & ((lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u));
}
// 0 times two bf16: 0, or NaN where one is not finite.
__device__ __forceinline__ uint32_t zero_times2(uint32_t v) {
    const bool lo = (v & 0x7f80u) == 0x7f80u, hi = (v & 0x7f800000u) == 0x7f800000u;
    return (lo ? 0x7fc0u : 0u) | (hi ? 0x7fc00000u : 0u);
}
// The larger magnitudes, halves apart, of two pairs of bf16 bits (`most`
// without signs); a half of 0x7f80 or more is not finite.
__device__ __forceinline__ uint32_t larger2(uint32_t most, uint32_t v) {
    typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, most),
                                                                  __builtin_bit_cast(u16x2_t, v & 0x7fff7fffu)));
}
__device__ __forceinline__ bool odd2(uint32_t most) { return (most & 0xffffu) >= 0x7f80u || (most >> 16) >= 0x7f80u; }

// Bits of keys y and y + 1 that lie in [lo, hi).
__device__ __forceinline__ uint32_t inside2(int y, int lo, int hi) {
    return (y >= lo && y < hi ? 0xffffu : 0u) | (y + 1 >= lo && y + 1 < hi ? 0xffff0000u : 0u);
}

// ------------------------------------------------------------ few query rows
//
// One workgroup per (tile of 16 query rows, KV head block, run of keys); its
// four waves take 32 keys (two pages) in turn, each with its own running
// maximum, sum and output, merged through LDS once at the end.  Keys and values
// go straight from the cache into the operands of the matrix products, the next
// 32 keys' loads in flight while the current ones are used:
//   S^T[key][q] = K[key][:] . Q[q][:]
//   O^T[dim][q] += V^T[dim][key] P^T[key][q]
// bf16: row 4 g + e of S's tile t (t = 0, 1) is key 8 g + 4 t + e of the 32, so
// that lane (q, g) ends with the keys 8 g .. 8 g + 7, exactly its operand of
// the second product, whose other operand is then one 16-byte load of the
// transposed V block.  fp32 (16 keys a product): the contraction's index g of
// step e is dimension 16 j + 4 g + e, or key 4 g + e, and row r of the output
// tile dt is dimension (D / 16) r + dt, all 16-byte loads again.
// bf16: probabilities are rounded to bf16, as the matrix product takes them, their
// sum is not (error against 64 bits 1.8e-3 to 1.9e-3 of the output, 1.6e-3 to
// 1.7e-3 with float32 probabilities, nearly all of it the output's own rounding).
// A second product with what the rounding left would take that away, but an
// infinite value times a remainder of 0 or below would end as NaN.
//
// What bounds it: HBM where there are many keys (32 single tokens over 512 to
// 16,384 keys, 1.1 GB: 210 us, 5.3 TB/s, what a large copy reaches; 220 us with
// the runs in the rows' order), the chain of loads lengths -> table -> keys and
// the second launch where there are few (4 tokens over 1075 keys of 16 heads 8.4
// us; with 16 waves a head in one launch 11.8 us: a CU alone draws 25 to 50 GB/s).
constexpr int NW = 4;

template <typename T, int D>
struct Keys;                                     // 32 keys in operand order

template <int D>
struct Keys<bf16_t, D> {
    uint4 k[2][D / 32];
    uint4 v[D / 16];
    __device__ __forceinline__ void load(const bf16_t* p0, const bf16_t* p1, size_t vofs, int r, int g) {
        // r >= 8: the second page's keys; g >= 2 likewise for V
        const bf16_t* kp = (r & 8 ? p1 : p0) + (8 * ((r >> 2) & 1) + (r & 3)) * D + 8 * g;
        const bf16_t* vp = (g & 2 ? p1 : p0) + vofs + r * PG + 8 * (g & 1);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int j = 0; j < D / 32; ++j) k[t][j] = *reinterpret_cast<const uint4*>(kp + 4 * t * D + 32 * j);
#pragma unroll
        for (int dt = 0; dt < D / 16; ++dt) v[dt] = *reinterpret_cast<const uint4*>(vp + 16 * dt * PG);
    }
};
template <int D>
struct Keys<float, D> {
    float4 k[2][D / 16];
    float4 v[2][4][D / 64];
    __device__ __forceinline__ void load(const float* p0, const float* p1, size_t vofs, int r, int g) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float* kp = (t ? p1 : p0) + r * D + 4 * g;
            const float* vp = (t ? p1 : p0) + vofs + 4 * g * D + (D / 16) * r;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) k[t][j] = *reinterpret_cast<const float4*>(kp + 16 * j);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < D / 64; ++i) v[t][e][i] = *reinterpret_cast<const float4*>(vp + e * D + 4 * i);
        }
    }
};

// Output dimension of accumulator (dt, e) of lane group g.
template <typename T, int D>
__device__ __forceinline__ int dim_of(int dt, int g, int e) {
    return sizeof(T) == 2 ? 16 * dt + 4 * g + e : (D / 16) * (4 * g + e) + dt;
}

template <typename T, int D>
__global__ __launch_bounds__(64 * NW, 2) void attn_rows_kernel(mtp_attention_args a, AttnGeo g) {
    constexpr int QR = 16, ND = D / 16;
    __shared__ __attribute__((aligned(16))) float s_acc[NW * QR * D];     // [wave][row][dimensions in order]
    __shared__ float s_m[NW][QR], s_l[NW][QR];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, gr = lane >> 4;
    const int H = a.cache.n_kv_heads, HB = H * g.hb;
    const int u = uniform(blockIdx.x / HB), hbi = blockIdx.x - u * HB, hk = hbi / g.hb;
    int tile, split;
    const AttnTile t = find_item(a, g, u, tile, split);
    if (t.nt == 0) return;
    int k0, k1;
    const int live = runs_of(g, t, split, k0, k1);
    if (split >= live) return;

    const int group = a.n_heads / H, h0 = (hbi - hk * g.hb) * g.gs;      // first head of the block in its group
    const int heads = min(g.gs, group - h0), rows = t.nt * g.gs;
    const int rc = r < rows && r % g.gs < heads ? r : 0;                  // rows that do not exist compute row 0
    const size_t vofs = (size_t)H * PG * D, pstr = 2 * vofs;
    const T* pool = (const T*)a.cache.pool + (size_t)hk * PG * D;
    const int32_t* tab = a.table + (size_t)t.c * a.max_pages;
    const int npairs = (k1 - k0 + 31) >> 5;                              // of the run
    const int mine = npairs > wave ? (npairs - wave + NW - 1) / NW : 0;  // of this wave: wave, wave + NW, ...
    // lane i: the pages of this wave's pair i (64 at a time); -1 where there is none
    int pg0 = -1, pg1 = -1;
    auto pages = [&](int i) {
        const int p = (k0 >> 4) + 2 * (wave + NW * (i + lane));
        int x = -1, y = -1;
        if (i + lane < mine) {
            x = p < a.max_pages ? tab[p] : -1;
            y = p + 1 < a.max_pages ? tab[p + 1] : -1;
        }
        pg0 = x >= 0 && x < a.cache.num_pages ? x : -1;
        pg1 = y >= 0 && y < a.cache.num_pages ? y : -1;
    };
    pages(0);                                                             // (before the queries' loads, as they return in order)
    const T* qp = (const T*)a.q + (int64_t)(t.t0 + rc / g.gs) * a.q_stride + (hk * group + h0 + rc % g.gs) * D;
    uint4 q[sizeof(T) == 2 ? D / 32 : D / 16];
#pragma unroll
    for (int j = 0; j < (sizeof(T) == 2 ? D / 32 : D / 16); ++j)
        q[j] = *reinterpret_cast<const uint4*>(qp + (sizeof(T) == 2 ? 32 * j + 8 * gr : 16 * j + 4 * gr));
    int rlo, rhi;
    sight_of(a, g, t, rc, rlo, rhi);
    // keys that every query of the tile sees: [alo, ahi)
    int alo, ahi, unused;
    sight_of(a, g, t, rows - 1, alo, unused);
    sight_of(a, g, t, 0, unused, ahi);
    const bool mixed = alo != t.lo || ahi != t.hi;       // some keys of the tile are seen by some of its queries only

    // (fp32 keys of 128 dimensions: 128 registers a set, one set only)
    constexpr int PD = sizeof(T) * D > 256 ? 1 : 2;
    Keys<T, D> kv[PD];
    int bad[PD] = {};                                                     // bit 0, 1: the pair's page is not there
    auto fetch = [&](Keys<T, D>& x, int& b, int i) {
        if ((i & 63) == 0 && i > 0) pages(i);
        const int x0 = __builtin_amdgcn_readlane(pg0, i & 63), x1 = __builtin_amdgcn_readlane(pg1, i & 63);
        b = (x0 < 0 ? 1 : 0) | (x1 < 0 ? 2 : 0);
        x.load(pool + (size_t)max(x0, 0) * pstr, pool + (size_t)max(x1, 0) * pstr, vofs, r, gr);
    };

    const float c = a.scale * LOG2E;
    float m = -INFINITY, l = 0.f;
    f32x4_t o[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    auto use = [&](Keys<T, D>& x, int b, int i) {
        const int kb = k0 + 32 * (wave + NW * i);
        // s[u]: bf16, keys kb + 8 gr + u; fp32, keys kb + 16 (u / 4) + 4 gr + u % 4
        float s[8];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int j = 0; j < D / 32; ++j)
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x.k[tt][j]),
                                                                  __builtin_bit_cast(bf16x8_t, q[j]), acc, 0, 0, 0);
            } else {
#pragma unroll
                for (int j = 0; j < D / 16; ++j) {
                    const float4 kk = x.k[tt][j], qq = __builtin_bit_cast(float4, q[j]);
                    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(kk.x, qq.x, acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(kk.y, qq.y, acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(kk.z, qq.z, acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(kk.w, qq.w, acc, 0, 0, 0);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) s[4 * tt + e] = acc[e] * c;
        }
        auto key_of = [&](int u) { return kb + (sizeof(T) == 2 ? 8 * gr + u : 16 * (u >> 2) + 4 * gr + (u & 3)); };
        auto there = [&](int u) {                                        // the key's page is in the pool
            return sizeof(T) == 2 ? !(b >> (gr >> 1) & 1) : !(b >> (u >> 2) & 1);
        };
        const bool edge = kb < alo || kb + 32 > ahi || kb + 32 > k1 || b;    // uniform
        bool odd = false;
        if (edge) {
            const int slo = max(rlo, t.lo), shi = min(rhi, k1);
#pragma unroll
            for (int u = 0; u < 8; ++u) s[u] = key_of(u) >= slo && key_of(u) < shi && there(u) ? s[u] : -INFINITY;
            // values that no query sees are not multiplied (0 x infinity, 0 x NaN); among those that some see and some
            // do not, the ones that are not finite are taken out here and added below
            if constexpr (sizeof(T) == 2) {
                uint32_t in[4], most = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) in[j] = there(0) ? inside2(kb + 8 * gr + 2 * j, t.lo, k1) : 0u;
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) {
                    uint4& v = x.v[dt];
                    v = make_uint4(v.x & in[0], v.y & in[1], v.z & in[2], v.w & in[3]);
                    most = larger2(larger2(larger2(larger2(most, v.x), v.y), v.z), v.w);
                }
                odd = mixed && odd2(most);
                if (__any(odd)) {
#pragma unroll
                    for (int dt = 0; dt < ND; ++dt) {
                        uint4& v = x.v[dt];
                        v = make_uint4(finite2(v.x), finite2(v.y), finite2(v.z), finite2(v.w));
                    }
                }
            } else {
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const bool in = key_of(u) >= t.lo && key_of(u) < k1 && there(u);
#pragma unroll
                    for (int i2 = 0; i2 < D / 64; ++i2) {
                        float* v = reinterpret_cast<float*>(&x.v[u >> 2][u & 3][i2]);
#pragma unroll
                        for (int d = 0; d < 4; ++d) {
                            const bool fin = !mixed || fabsf(v[d]) < INFINITY;
                            odd |= in && !fin;
                            v[d] = in && fin ? v[d] : 0.f;
                        }
                    }
                }
            }
        }
        float mx = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
        mx = xor16_max(mx);
        mx = xor32_max(mx);
        if (__any(mx > m)) {
            const float mn = fmaxf(m, mx), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= f;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) o[dt] *= f;
        }
        const float mm = m == -INFINITY ? 0.f : m;
        float p[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) p[u] = __builtin_amdgcn_exp2f(s[u] - mm);
        l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
        if constexpr (sizeof(T) == 2) {
            const bf16x8_t pf = __builtin_bit_cast(
                bf16x8_t, make_uint4(pk2(p[0], p[1]), pk2(p[2], p[3]), pk2(p[4], p[5]), pk2(p[6], p[7])));
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
                o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x.v[dt]), pf, o[dt], 0, 0, 0);
        } else {
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int dt = 0; dt < ND; ++dt)
                    o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                        reinterpret_cast<const float*>(&x.v[u >> 2][u & 3][0])[dt], p[u], o[dt], 0, 0, 0);
        }
        if (__any(odd)) {
            // an infinite or NaN value reaches exactly the queries that see it
            const int pr = wave + NW * i;
            for (int u = 0; u < 32; ++u) {
                const int key = kb + u, at = (k0 >> 4) + 2 * pr + (u >> 4);
                if (key >= k1 || key < t.lo || (b >> (u >> 4) & 1)) continue;
                const T* vb = pool + (size_t)tab[at] * pstr + vofs;
                const bool sees = key >= rlo && key < rhi;
#pragma unroll
                for (int dt = 0; dt < ND; ++dt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int d = dim_of<T, D>(dt, gr, e);
                        const float v = ActIO<T>::load(vb + (sizeof(T) == 2 ? d * PG + (u & 15) : (u & 15) * D + d));
                        if (sees && !(fabsf(v) < INFINITY)) o[dt][e] += v;
                    }
            }
        }
    };

    if constexpr (PD == 1) {
        for (int i = 0; i < mine; ++i) {
            fetch(kv[0], bad[0], i);
            use(kv[0], bad[0], i);
        }
    } else {
        if (mine > 0) fetch(kv[0], bad[0], 0);
        for (int i = 0; i < mine; i += 2) {
            if (i + 1 < mine) fetch(kv[1], bad[1], i + 1);
            use(kv[0], bad[0], i);
            if (i + 1 < mine) {
                if (i + 2 < mine) fetch(kv[0], bad[0], i + 2);
                use(kv[1], bad[1], i + 1);
            }
        }
    }
    l = xor16_sum(l);
    l = xor32_sum(l);

    // merge the waves
    if (gr == 0) { s_m[wave][r] = m; s_l[wave][r] = l; }
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<f32x4_t*>(&s_acc[(wave * QR + r) * D + 16 * dt + 4 * gr]) = o[dt];
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) s_acc[(wave * QR + r) * D + dim_of<T, D>(dt, gr, e)] = o[dt][e];
        }
    }
    __syncthreads();
    const size_t slot = (((size_t)tile * HB + hbi) * g.n_splits + split) * QR;
    for (int i = threadIdx.x; i < rows * (D / 4); i += 64 * NW) {
        const int qr = i / (D / 4), d = (i - qr * (D / 4)) * 4;
        if (qr % g.gs >= heads) continue;
        float mm = s_m[0][qr];
#pragma unroll
        for (int w = 1; w < NW; ++w) mm = fmaxf(mm, s_m[w][qr]);
        float ll = 0.f;
        f32x4_t v = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = s_m[w][qr] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_m[w][qr] - mm);
            ll += f * s_l[w][qr];
            const f32x4_t ow = *reinterpret_cast<const f32x4_t*>(&s_acc[(w * QR + qr) * D + d]);
            v += ow * f;
        }
        if (live > 1) {
            *reinterpret_cast<f32x4_t*>(&g.acc[(slot + qr) * D + d]) = v;
            if (d == 0) g.ml[slot + qr] = make_float2(mm, ll);
        } else {
            // (a row that sees nothing has a sum of 0; one whose scores are not numbers keeps that)
            const float inv = ll == 0.f ? 0.f : 1.f / ll;
            T* op = (T*)a.out + (int64_t)(t.t0 + qr / g.gs) * a.out_stride + (hk * group + h0 + qr % g.gs) * D + d;
            if constexpr (sizeof(T) == 2)
                *reinterpret_cast<uint2*>(op) = make_uint2(pk2(v[0] * inv, v[1] * inv), pk2(v[2] * inv, v[3] * inv));
            else
                *reinterpret_cast<f32x4_t*>(op) = v * inv;
        }
    }
}

// ----------------------------------------------------------- many query rows
//
// One workgroup per (tile of 128 query rows, KV head block, run of keys) for
// bf16 caches: four waves of 32 query rows each over blocks of 64 keys (four
// pages) that they share through LDS, the next block's loads going straight to
// LDS while the current one is used.
//   S^T[key][q] = K[key][:] . Q[q][:]       32 x 32 x 16 products
//   O^T[dim][q] += V^T[dim][key] P^T[key][q]
// Row 16 s + 8 j + 4 h + e of a 32-key tile of S is key 16 s + 8 h + 4 j + e, so
// that lane (q, h) holds the keys 16 s + 8 h .. + 7 in its registers 8 s .. 8 s
// + 7: its operand of the second product, the other one being 16 bytes of a V
// page.  K rows and V pages are whole multiples of the banks, so their 16-byte
// pieces are stored in an order that slot and dimension shift (the address that
// a lane loads from, not where it stores): 16 lanes then read 16 different
// banks' pieces.
// The reference m moves only when a score exceeds it by 8 (float32 sums and
// bf16 probabilities up to 2^8 keep their relative precision).  Probabilities
// are rounded to bf16, as the matrix product takes them; their sum is not.
// Blocks that every query of the tile sees whole run in a loop of their own,
// without masks: in one loop with the others the accumulators were copied every
// block (367 us instead of 320 us below).
//
// What bounds it: the matrix cores and the vector unit in turn.  A block costs a
// wave 1000 cycles of products and as many of exponentials, maxima, sums and
// conversions; counters show each busy 42 to 44% of the time, the two waves of a
// SIMD overlapping little.  Forming the next block's scores during the
// exponentials (software pipelining) measured the same and cost registers; so
// did a third block in LDS, raised priority around the products, and sums by dot
// products of the rounded probabilities.  Measured, 32 query heads on 8 KV heads
// of 128: chunks of 512 tokens over 8192 keys 302 us (880 TFLOP/s), whole prompts
// of 4096 620 us (887), chunks of 400 to 512 over 2048 to 8192 keys in any order
// 192 to 210 us (196 to 233 in the rows' order; 12 us of it the join); 16 heads of
// 64, 8 prompts of 450 tokens 20.2 us.  Pages of a part-seen block that no row of
// the wave sees are left out, scores and values: chunks over 8192 keys 302 us
// instead of 314 us.
// Head dim 64 with four workgroups a CU instead of three: 230 -> 199 us.  It has
// 128 registers a lane for them and spills 7 (32 bytes of scratch), stored once
// before the loops; blocks at the edge of what is seen read some of them back and
// a refill of the page numbers one, the loop over whole blocks none.
constexpr int TR = 128;                          // query rows of a tile
constexpr int KB = 64;                           // keys of a block

typedef const __attribute__((address_space(1))) void* gptr_t;
typedef __attribute__((address_space(3))) void* lptr_t;

// ZERO: scale 0, in a kernel of its own (as a branch in one kernel it cost every call 4 to 20%, by the registers around it).
template <int D, bool ZERO>
__global__ __launch_bounds__(256, D == 64 ? 4 : 2) void attn_tile_kernel(mtp_attention_args a, AttnGeo g) {
    constexpr float MSTEP = 8.0f;
    constexpr int CW = D / 8;                    // 16-byte pieces of a K row
    __shared__ __attribute__((aligned(1024))) bf16_t s_k[2][KB * D], s_v[2][KB * D];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int qc = lane & 31, hh = lane >> 5;
    const int H = a.cache.n_kv_heads, HB = H * g.hb;
    // heads fastest: workgroups are dealt to the 8 XCDs in turn, so that with a multiple of 8 heads each XCD has its own,
    // whose keys its L2 then holds
    const int u = uniform(blockIdx.x / HB), hbi = blockIdx.x - u * HB, hk = hbi / g.hb;
    int tile, split;
    const AttnTile t = find_item(a, g, u, tile, split);
    if (t.nt == 0) return;
    int k0, k1;
    const int live = runs_of(g, t, split, k0, k1);
    if (split >= live) return;

    const int group = a.n_heads / H, h0 = (hbi - hk * g.hb) * g.gs;
    const int heads = min(g.gs, group - h0), rows = t.nt * g.gs;
    const bool wave_on = 32 * wave < rows;       // uniform
    const int r0 = min(32 * wave, rows - 1), r1 = min(32 * wave + 31, rows - 1);
    const int row = min(32 * wave + qc, r1);
    const int hq = row % g.gs < heads ? row % g.gs : 0;   // heads that do not exist compute the block's first
    const size_t vofs = (size_t)H * PG * D, pstr = 2 * vofs;
    const bf16_t* pool = (const bf16_t*)a.cache.pool + (size_t)hk * PG * D;
    const int32_t* tab = a.table + (size_t)t.c * a.max_pages;
    const int nb = k1 > k0 ? (k1 - k0 + KB - 1) / KB : 0;
    const int pg_end = min(a.max_pages, (k1 + PG - 1) / PG);
    // lane i: page i of the next 64 (16 blocks), -1 where there is none
    auto pages = [&](int blk) {
        const int p = k0 / PG + 4 * blk + lane;
        const int x = p < pg_end ? tab[p] : -1;
        return x >= 0 && x < a.cache.num_pages ? x : -1;
    };
    // (before the queries' loads: loads return in order, and the keys' wait for these)
    int pg_now = pages(0), pg_next = pages(16);
    const bf16_t* qp = (const bf16_t*)a.q + (int64_t)(t.t0 + row / g.gs) * a.q_stride + (hk * group + h0 + hq) * D + 8 * hh;
    // scores are S x c with c > 0: a negative scale turns the queries' signs, scale 0 (ZERO) their values to 0 times them
    const float c = ZERO ? 1.f : fabsf(a.scale) * LOG2E;
    bf16x8_t q[D / 16];
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
        u32x4_t v = *reinterpret_cast<const u32x4_t*>(qp + 16 * j);
        if (ZERO) v = u32x4_t{zero_times2(v[0]), zero_times2(v[1]), zero_times2(v[2]), zero_times2(v[3])};
        else if (a.scale < 0.f) v ^= 0x80008000u;
        q[j] = __builtin_bit_cast(bf16x8_t, v);
    }
    // what this lane's row sees; what some row of the wave sees; what every row of the tile sees
    int rlo, rhi, wlo, whi, tlo, thi, skip;
    sight_of(a, g, t, row, rlo, rhi);
    sight_of(a, g, t, r0, wlo, skip);
    sight_of(a, g, t, r1, skip, whi);
    sight_of(a, g, t, 0, skip, thi);
    sight_of(a, g, t, rows - 1, tlo, skip);
    const bool mixed = tlo != t.lo || thi != t.hi;       // some keys of the tile are seen by some of its queries only

    // what each lane loads of a page in one step: K's piece of slot `slot`, V's in order
    constexpr int SPP = D / 32;                  // wave steps (1 KB) per page block
    auto stage = [&](int buf, int blk) {
        if ((blk & 15) == 0 && blk > 0) { pg_now = pg_next; pg_next = pages(blk + 16); }
        int bad = 0;
#pragma unroll
        for (int p = 0; p < 4; ++p)
            bad |= __builtin_amdgcn_readlane(pg_now, 4 * (blk & 15) + p) < 0 ? 1 << p : 0;
#pragma unroll
        for (int i = 0; i < SPP; ++i) {
            const int step = 4 * i + wave, p = step / SPP, in = (step % SPP) * 64 + lane;
            const int pg = max(__builtin_amdgcn_readlane(pg_now, 4 * (blk & 15) + p), 0);
            const bf16_t* base = pool + (size_t)pg * pstr;
            const int slot = in / CW, piece = (in % CW) ^ (D == 128 ? slot : (slot >> 1) & 7);
            __builtin_amdgcn_global_load_lds((gptr_t)(base + slot * D + piece * 8), (lptr_t)(&s_k[buf][step * 512]), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((gptr_t)(base + vofs + (in ^ ((in >> 4) & 1)) * 8), (lptr_t)(&s_v[buf][step * 512]),
                                             16, 0, 0);
        }
        return bad;
    };

    float m = -INFINITY, l = 0.f;
    f32x16_t o[D / 32];
#pragma unroll
    for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;

    // K operand: row qc of a tile is key krow
    const int krow = (qc & 16) | ((qc & 4) << 1) | ((qc & 8) >> 1) | (qc & 3);
    const int ksw = D == 128 ? krow & 15 : (krow >> 1) & 7;

    // the scores of the block in buffer buf
    auto scores = [&](int buf, f32x16_t (&s)[2]) {
        const bf16_t* K = s_k[buf] + krow * D;
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[tt][i] = 0.f;
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
                s[tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    *reinterpret_cast<const bf16x8_t*>(K + 32 * tt * D + ((2 * j + hh) ^ ksw) * 8), q[j], s[tt], 0, 0, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int i = 0; i < D / 8 - 4; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    };
    // their probabilities; m, l and o move along
    auto weigh = [&](const f32x16_t (&s)[2], bf16x8_t (&p)[4]) {
        float mx = -INFINITY;
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[tt][i]);
        mx *= c;
        if (__any(mx > (m == -INFINITY ? -INFINITY : m + MSTEP))) {
            mx = xor32_max(mx);
            const float mn = fmaxf(m, mx), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= f;
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt) o[dt] *= f;
        }
        const float mm = m == -INFINITY ? 0.f : m;
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = __builtin_amdgcn_exp2f(fmaf(s[u >> 1][8 * (u & 1) + i], c, -mm));
            sum += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
            p[u] = __builtin_bit_cast(bf16x8_t, make_uint4(pk2(e[0], e[1]), pk2(e[2], e[3]), pk2(e[4], e[5]), pk2(e[6], e[7])));
        }
        l += sum;
    };
    // a block that every query of the tile sees whole
    auto whole = [&](int buf) {
        f32x16_t s[2];
        bf16x8_t p[4];
        scores(buf, s);
        weigh(s, p);
        const bf16_t* V = s_v[buf] + qc * PG + 8 * (hh ^ ((qc >> 3) & 1));
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt)
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    *reinterpret_cast<const bf16x8_t*>(V + u * PG * D + 32 * dt * PG), p[u], o[dt], 0, 0, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (int i = 0; i < D / 8 - 4; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    };
    // any block
    auto edge = [&](int buf, int kb, int bad) {
        f32x16_t s[2];
        bf16x8_t p[4];
        const int end = min(k1, whi);            // no row of the wave sees keys from here on, nor before wlo
        if (kb + 32 < end) {
            scores(buf, s);
        } else {
            const bf16_t* K = s_k[buf] + krow * D;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[0][i] = s[1][i] = 0.f;
#pragma unroll
            for (int j = 0; j < D / 16; ++j)
                s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                    *reinterpret_cast<const bf16x8_t*>(K + ((2 * j + hh) ^ ksw) * 8), q[j], s[0], 0, 0, 0);
        }
        // register i of tile tt: key kb + 32 tt + 16 (i / 8) + 8 hh + i % 8, page 2 tt + i / 8 of the block
        const int slo = max(rlo, t.lo) - (kb + 8 * hh);
        const unsigned span = max(0, min(rhi, k1) - max(rlo, t.lo));
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                s[tt][i] = (unsigned)(32 * tt + 16 * (i >> 3) + (i & 7) - slo) < span ? s[tt][i] : -INFINITY;
        if (bad) {
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[tt][i] = bad >> (2 * tt + (i >> 3)) & 1 ? -INFINITY : s[tt][i];
        }
        weigh(s, p);
        const bf16_t* V = s_v[buf] + qc * PG + 8 * (hh ^ ((qc >> 3) & 1));
        // values that no query sees are not multiplied (0 x infinity, 0 x NaN); among those that some see and some
        // do not, the ones that are not finite are taken out here and added below
        bool odd = false;
        if (mixed) {
            uint32_t most = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt) {
                    const uint4 v = *reinterpret_cast<const uint4*>(V + u * PG * D + 32 * dt * PG);
                    most = larger2(larger2(larger2(larger2(most, v.x), v.y), v.z), v.w);
                }
            odd = odd2(most);                    // (of keys outside [t.lo, k1) too: those come to nothing below)
        }
        const bool any_odd = __any(odd);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            // the page's first key: uniform, as the ways below are (with head dim 64 there are no registers for the
            // second: 16 rows of 450 tokens 34 us with it, 28.5 us without)
            const int ka = kb + 16 * u;
            if ((bad >> u & 1) || ka >= end || ka + PG <= wlo) continue;
            if (D == 128 && ka >= t.lo && ka + PG <= k1 && !any_odd) {
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt)
                    o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        *reinterpret_cast<const bf16x8_t*>(V + u * PG * D + 32 * dt * PG), p[u], o[dt], 0, 0, 0);
                continue;
            }
            uint32_t in[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) in[j] = inside2(ka + 8 * hh + 2 * j, t.lo, k1);
#pragma unroll
            for (int dt = 0; dt < D / 32; ++dt) {
                uint4 v = *reinterpret_cast<const uint4*>(V + u * PG * D + 32 * dt * PG);
                v = make_uint4(v.x & in[0], v.y & in[1], v.z & in[2], v.w & in[3]);
                if (any_odd) v = make_uint4(finite2(v.x), finite2(v.y), finite2(v.z), finite2(v.w));
                o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, v), p[u], o[dt], 0, 0, 0);
            }
        }
        if (any_odd) {
            // an infinite or NaN value reaches exactly the queries that see it
            for (int u = 0; u < KB; ++u) {
                const int key = kb + u;
                if (key >= k1 || key < t.lo || (bad >> (u >> 4) & 1)) continue;
                const bool sees = key >= rlo && key < rhi;
#pragma unroll
                for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int d = 32 * dt + 8 * (i >> 2) + 4 * hh + (i & 3);
                        const float v = bf16_to_f32(s_v[buf][(u >> 4) * PG * D + d * PG + ((u & 15) ^ (d & 8))]);
                        if (sees && !(fabsf(v) < INFINITY)) o[dt][i] += v;
                    }
            }
        }
    };

    // blocks [w0, w1) are seen whole by every query of the tile
    const int w0 = max(0, (tlo - k0 + KB - 1) / KB), w1 = (min(thi, k1) - k0) / KB;
    int bad = nb > 0 ? stage(0, 0) : 0;
    int j = 0;
    // this wave's loads of block j have landed; all waves' have, and all are done with block j - 1's buffer
    auto arrive = [&]() {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const int now = bad;
        if (j + 1 < nb) bad = stage((j + 1) & 1, j + 1);
        return now;
    };
    while (j < nb) {
        for (; j >= w0 && j < w1 && bad == 0; ++j) {
            arrive();
            if (wave_on) whole(j & 1);
        }
        if (j < nb) {
            const int now = arrive(), kb = k0 + KB * j;
            if (wave_on && kb < whi && kb + KB > wlo) edge(j & 1, kb, now);
            ++j;
        }
    }
    l = xor32_sum(l);

    const int qr = 32 * wave + qc;
    if (qr >= rows || qr % g.gs >= heads) return;
    // register i of o[dt]: dimension 32 dt + 8 (i / 4) + 4 hh + i % 4
    if (live > 1) {
        const size_t slot = (((size_t)tile * HB + hbi) * g.n_splits + split) * TR + qr;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<f32x4_t*>(&g.acc[slot * D + 32 * dt + 2 * i + 4 * hh]) =
                    f32x4_t{o[dt][i], o[dt][i + 1], o[dt][i + 2], o[dt][i + 3]};
        if (hh == 0) g.ml[slot] = make_float2(m, l);
    } else {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        bf16_t* op = (bf16_t*)a.out + (int64_t)(t.t0 + qr / g.gs) * a.out_stride + (hk * group + h0 + qr % g.gs) * D + 8 * hh;
#pragma unroll
        for (int dt = 0; dt < D / 32; ++dt)
#pragma unroll
            for (int i = 0; i < 16; i += 8) {
                // of 16 dimensions lane h has 4 h .. + 3 and 8 + 4 h .. + 3; exchanged, 8 h .. + 7
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = pk2(o[dt][i + 2 * k] * inv, o[dt][i + 2 * k + 1] * inv);
                const auto x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
                const auto y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
                *reinterpret_cast<uint4*>(op + 32 * dt + 2 * i) = make_uint4(x[0], y[0], x[1], y[1]);
            }
    }
}

// Joins a tile's runs: one wave per JR query rows, whose loads are in flight
// together.  The runs' weights exp2(m_s - m) once (lane i: runs i, i + 64, ...),
// then every group of D / 4 lanes takes runs in turn.
constexpr int JW = 4;                            // waves of a workgroup

constexpr int JFEW = 4;                          // runs up to which a wave takes four rows

template <typename T, int D, int RT, int JR>
__global__ __launch_bounds__(64 * JW) void attn_join_kernel(mtp_attention_args a, AttnGeo g) {
    constexpr int NL = JR == 1 ? MAX_RUNS / 64 : 1;    // runs of a lane
    constexpr int LD = D / 4, SG = 64 / LD;      // lanes of a row's dimensions, runs at a time
    __shared__ float s_w[JW][JR][64 * NL];
    const int H = a.cache.n_kv_heads, HB = H * g.hb, lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tile = blockIdx.x / HB, hbi = blockIdx.x - tile * HB, hk = hbi / g.hb, q0 = (blockIdx.y * JW + wave) * JR;
    const AttnTile t = find_tile(a, g, tile);
    const int group = a.n_heads / H, h0 = (hbi - hk * g.hb) * g.gs, heads = min(g.gs, group - h0), rows = t.nt * g.gs;
    if (q0 >= rows) return;
    int k0, k1;
    const int live = runs_of(g, t, 0, k0, k1);
    if (live <= 1) return;
    const size_t slot = (size_t)blockIdx.x * g.n_splits * RT + q0;
    // (a run that the row sees nothing of has m = -infinity and l = 0; one whose scores are not numbers l = NaN; rows
    // that do not exist read the first one's)
    float2 x[JR][NL];
    float m[JR], l[JR];
#pragma unroll
    for (int k = 0; k < JR; ++k)
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            x[k][i] = make_float2(-INFINITY, 0.f);
            if (64 * i + lane < live) x[k][i] = g.ml[slot + (q0 + k < rows ? k : 0) + (size_t)(64 * i + lane) * RT];
        }
#pragma unroll
    for (int k = 0; k < JR; ++k) {
        m[k] = -INFINITY;
        l[k] = 0.f;
#pragma unroll
        for (int i = 0; i < NL; ++i) m[k] = fmaxf(m[k], x[k][i].x);
        m[k] = wave_max64(m[k]);
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const float w = x[k][i].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x[k][i].x - m[k]);
            l[k] += x[k][i].x == -INFINITY ? x[k][i].y : w * x[k][i].y;
            s_w[wave][k][64 * i + lane] = w;
        }
        l[k] = wave_sum64(l[k]);
    }
    __builtin_amdgcn_wave_barrier();
    const int sg = lane / LD, d = (lane - sg * LD) * 4;
    f32x4_t v[JR];
#pragma unroll
    for (int k = 0; k < JR; ++k) v[k] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll JR == 1 ? 8 : 2
    for (int s = sg; s < live; s += SG) {
#pragma unroll
        for (int k = 0; k < JR; ++k) {
            const float w = s_w[wave][k][s];
            const f32x4_t o =
                *reinterpret_cast<const f32x4_t*>(&g.acc[(slot + (q0 + k < rows ? k : 0) + (size_t)s * RT) * D + d]);
            v[k] += o * w;                       // (0 x infinity: an infinite value that is seen shows)
        }
    }
#pragma unroll
    for (int k = 0; k < JR; ++k) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (LD == 16) v[k][e] = xor16_sum(v[k][e]);
            v[k][e] = xor32_sum(v[k][e]);
        }
        const int qr = q0 + k;
        if (sg != 0 || qr >= rows || qr % g.gs >= heads) continue;
        const float inv = l[k] == 0.f ? 0.f : 1.f / l[k];
        T* op = (T*)a.out + (int64_t)(t.t0 + qr / g.gs) * a.out_stride + (hk * group + h0 + qr % g.gs) * D + d;
        if constexpr (sizeof(T) == 2)
            *reinterpret_cast<uint2*>(op) = make_uint2(pk2(v[k][0] * inv, v[k][1] * inv), pk2(v[k][2] * inv, v[k][3] * inv));
        else
            *reinterpret_cast<f32x4_t*>(op) = v[k] * inv;
    }
}

// ------------------------------------------------------------------- launches
// (Four rows a wave where there are few runs: two runs of 488 wide tiles 28 us with one row a wave, 15 us; many
// runs of few tiles are faster with a row each: 11 runs of 48 wide tiles, the whole call 51.5 and 41 us.)
template <typename T, int D, int RT>
void join_go(hipStream_t st, const mtp_attention_args& a, const AttnGeo& g, unsigned work) {
    if (g.n_splits <= 1) return;
    const int rows = g.tt * g.gs;
    if (g.n_splits <= JFEW)
        hipLaunchKernelGGL((attn_join_kernel<T, D, RT, 4>), dim3(work, (rows + 4 * JW - 1) / (4 * JW)), dim3(64 * JW), 0, st, a, g);
    else
        hipLaunchKernelGGL((attn_join_kernel<T, D, RT, 1>), dim3(work, (rows + JW - 1) / JW), dim3(64 * JW), 0, st, a, g);
}

template <typename T, int D>
int rows_go(hipStream_t st, const mtp_attention_args& a, const AttnGeo& g) {
    const unsigned work = (unsigned)(g.n_tiles * a.cache.n_kv_heads * g.hb);
    hipLaunchKernelGGL((attn_rows_kernel<T, D>), dim3(work * g.n_splits), dim3(64 * NW), 0, st, a, g);
    join_go<T, D, 16>(st, a, g, work);
    return hipGetLastError() == hipSuccess ? MTP_OK : MTP_EHIP;
}

template <int D>
int tile_go(hipStream_t st, const mtp_attention_args& a, const AttnGeo& g) {
    const unsigned work = (unsigned)(g.n_tiles * a.cache.n_kv_heads * g.hb);
    if (a.scale == 0.f) hipLaunchKernelGGL((attn_tile_kernel<D, true>), dim3(work * g.n_splits), dim3(256), 0, st, a, g);
    else hipLaunchKernelGGL((attn_tile_kernel<D, false>), dim3(work * g.n_splits), dim3(256), 0, st, a, g);
    join_go<bf16_t, D, TR>(st, a, g, work);
    return hipGetLastError() == hipSuccess ? MTP_OK : MTP_EHIP;
}

// The cut of a call: kernel, tile shape, runs and the workspace of the partial
// sums.
struct AttnCut { AttnGeo g; bool wide; uint64_t acc_bytes, bytes; };

// (of a call with rows and tokens)
AttnCut attn_cut(const mtp_attention_args& a) {
    AttnCut x{};
    const int group = a.n_heads / a.cache.n_kv_heads;
    x.g.hb = (group + 15) / 16;
    x.g.gs = (group + x.g.hb - 1) / x.g.hb;
    // the most keys that a query sees, as far as the host knows
    int64_t kv = (int64_t)PG * a.max_pages;
    if (a.max_kv > 0) kv = std::min<int64_t>(kv, a.max_kv);
    if (a.window > 0) kv = std::min<int64_t>(kv, a.window);
    // The wide kernel from this many query rows a cache row on (16 rows, 8 KV heads, 1000 to 4000 keys from HBM: head dim
    // 128, 8 rows 41.5 us wide and 58.9 us narrow; head dim 64, 64 rows 55 and 57 us, 48 rows 57 and 46 us), where the
    // work is past its latency.  That is counted in pairs of a 16-row tile and a key: 250,000 with head dim 128 (one
    // sequence of 32 tokens over 4000 keys, 32 heads on 8, 256,000 pairs: 17.6 us wide and 20.1 us narrow; of 8 tokens
    // over 1000 keys, 8 heads on 2, 4000 pairs: 18 and 11 us), 500,000 with 64 (4 sequences of 32 tokens, 32 heads on 8:
    // 1000 keys, 256,000 pairs, 18 and 11 us; 4000 keys, a million, 25 us either way).
    const bool d128 = a.cache.head_dim == 128;
    const int64_t query_rows = (int64_t)a.n_tokens * x.g.gs;
    const int64_t pairs = std::max<int64_t>(a.n_rows, query_rows / 16) * a.cache.n_kv_heads * x.g.hb * kv;
    x.wide = a.cache.dtype == MTP_DTYPE_BF16 && query_rows >= (d128 ? 8ll : 64ll) * a.n_rows &&
             pairs >= (d128 ? 250000ll : 500000ll);
    const int rt = x.wide ? TR : 16;
    x.g.tt = rt / x.g.gs;
    x.g.n_tiles = a.n_rows == 1 ? (a.n_tokens + x.g.tt - 1) / x.g.tt : a.n_tokens / x.g.tt + a.n_rows;
    const int64_t work = (int64_t)x.g.n_tiles * a.cache.n_kv_heads * x.g.hb;
    // the most that a tile sees (32 single tokens of up to 16,384 keys in a window of 1024: 26 us, 36 us cut as if they
    // saw all)
    if (a.window > 0) kv = std::min<int64_t>(kv + x.g.tt + 31, (int64_t)PG * a.max_pages);
    // Sorting costs a workgroup some 25 ns a row, more than it gives few query rows on short keys (40 single tokens over
    // up to 700 keys, 16 heads: 19.1 us in the tiles' order, 20.1 us sorted; 32 over up to 1190 keys 27.8 and 27.0 us;
    // wide, 16 rows of 300 to 750 tokens over up to 150: 21.4 and 20.5 us).
    x.g.sorted = a.n_rows > 1 && a.n_rows <= 64 && (x.wide || kv >= 20ll * a.n_rows);
    // Runs of the keys.  Wide: 512 workgroups, two a CU, as many as fit with head dim 128; 768 with head dim 64 (16 rows
    // of 128 tokens: 45.4 us, 52 us with 1152) and where the tiles are part full (16 rows of 8 query rows over 1000 to
    // 4000 keys, head dim 128: 43 us, 49 us with 512).  With
    // head dim 64 and full tiles up to four runs, for the sorted order's sake (6 rows of 300 to 512 tokens over up to
    // 8192 keys: two runs 93 us, three 79; 3 rows of 64 to 600 over up to 6000: four 51 us, five 60).  No run shorter
    // than 256 keys.  Narrow: 512 workgroups, runs of 128 keys at least, at most 32 of them (16,000 keys of 8 KV heads 26
    // us, 33 us in 64); whole below 512 keys (400 keys of 16 heads 7.4 us, 8.1 us in three runs) and where the tiles fill
    // three quarters of the CUs (8 rows of up to 3650 keys, 240 tiles, 34.5 us, 38 us in three) or, below 2048 keys, a
    // third (16 rows of 16 tokens over 1000 keys, 8 heads of 64 on 2, 160 tiles, 11 us, 15 us in four).  But runs of 1024 keys of
    // long caches, which even out ragged rows, while the tiles are part full, up to ten workgroups a CU (8 rows of 32
    // tokens over 3000 to 8000 keys, 8 heads of 64: 54 us whole, 34 us in seven; 32 single tokens over up to 16,384: 242
    // us in two, 210 in eight, 225 in twelve).
    const bool few = (int64_t)a.n_tokens * x.g.gs <= (int64_t)TR * a.n_rows;
    int64_t n;
    auto runs = [&](int64_t workgroups) { return (workgroups + work - 1) / work; };
    if (x.wide) {
        n = runs(few || !d128 ? 768 : 512);
        if (!few && !d128) n = std::max<int64_t>(n, std::min<int64_t>(runs(1152), 4));
        n = std::min<int64_t>(n, kv / 256);
    } else {
        n = kv < 512 || work >= (kv < 2048 ? 96 : 192) ? 1 : std::min<int64_t>(std::min<int64_t>(runs(512), kv / 128), 32);
        if (kv >= 4096 && few) n = std::max<int64_t>(n, std::min<int64_t>(kv / 1024, 2560 / work));
    }
    n = std::max<int64_t>(1, std::min<int64_t>(n, MAX_RUNS));
    x.g.n_splits = (int)n;
    x.g.split_len = (int)(((kv + n - 1) / n + KB - 1) / KB * KB);
    if (n > 1) {
        x.acc_bytes = (uint64_t)work * n * rt * a.cache.head_dim * 4;
        x.bytes = x.acc_bytes + (uint64_t)work * n * rt * 8;
    }
    return x;
}

bool aligned(const void* p, uintptr_t n) { return p && ((uintptr_t)p & (n - 1)) == 0; }

int attn_check(const mtp_attention_args* a) {
    if (!a) return MTP_EINVAL;
    const int rc = cache_check(a->cache);
    if (rc != MTP_OK) return rc;
    if (a->n_rows < 0 || a->n_rows > 4096 || a->max_pages < 1 || a->max_pages > 65536 || a->n_tokens < 0 ||
        a->n_tokens >= (1 << 24) || a->n_heads < 1 || a->n_heads > 1024 || a->n_heads % a->cache.n_kv_heads)
        return MTP_EINVAL;
    // (a launch holds fewer than 2^32 threads, so fewer than 2^24 workgroups: two tiles of 16 hold at least 17 query
    // rows, the last tiles of the cache rows, part full, come to at most 4096 x 1024)
    if ((int64_t)(a->n_tokens + a->n_rows) * a->n_heads >= (1ll << 27)) return MTP_EINVAL;
    if (a->mode != MTP_ATTN_CAUSAL && a->mode != MTP_ATTN_FULL) return MTP_EINVAL;
    if (a->window < 0 || (a->mode == MTP_ATTN_FULL && a->window != 0) || a->max_kv < 0 || !isfinite(a->scale * LOG2E))
        return MTP_EINVAL;
    return MTP_OK;
}

}  // namespace
}  // namespace mtp

extern "C" {

int mtp_pages_attention_workspace_size(const mtp_attention_args* args, uint64_t* bytes) {
    const int rc = mtp::attn_check(args);
    if (rc != MTP_OK || !bytes) return MTP_EINVAL;
    *bytes = args->n_rows == 0 || args->n_tokens == 0 ? 0 : mtp::attn_cut(*args).bytes;
    return MTP_OK;
}

int mtp_pages_attention(const mtp_attention_args* args, void* hip_stream) {
    using namespace mtp;
    const int rc = attn_check(args);
    if (rc != MTP_OK) return rc;
    mtp_attention_args a = *args;
    if (a.n_rows == 0 || a.n_tokens == 0) return MTP_OK;
    // (a window of all that a row can hold hides nothing, and a larger one would carry the first position that a query
    // before the row's start sees, pos - window + 1, out of 32 bits)
    a.window = std::min(a.window, PG * a.max_pages);
    const int64_t per = a.cache.dtype == MTP_DTYPE_BF16 ? 8 : 4, row = (int64_t)a.n_heads * a.cache.head_dim;
    if (!aligned(a.table, 4) || !aligned(a.row_start, 4) || !aligned(a.kv_len, 4) || !aligned(a.q, 16) ||
        !aligned(a.out, 16) || a.q_stride < row || a.out_stride < row || a.q_stride % per || a.out_stride % per)
        return MTP_EINVAL;
    AttnCut x = attn_cut(a);
    if (x.bytes) {
        if (!aligned(a.workspace, 256)) return MTP_EINVAL;
        if (a.workspace_bytes < x.bytes) return MTP_ENOMEM;
        x.g.acc = (float*)a.workspace;
        x.g.ml = (float2*)((char*)a.workspace + x.acc_bytes);
    }
    hipStream_t st = (hipStream_t)hip_stream;
    const bool bf = a.cache.dtype == MTP_DTYPE_BF16;
    if (x.wide) return a.cache.head_dim == 64 ? tile_go<64>(st, a, x.g) : tile_go<128>(st, a, x.g);
    if (a.cache.head_dim == 64) return bf ? rows_go<bf16_t, 64>(st, a, x.g) : rows_go<float, 64>(st, a, x.g);
    return bf ? rows_go<bf16_t, 128>(st, a, x.g) : rows_go<float, 128>(st, a, x.g);
}

}  // extern "C"
