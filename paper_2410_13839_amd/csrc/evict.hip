// Eviction from a paged cache by accumulated attention weight
// (mtp_pages_evict).  See include/mtp.h for the operator's definition.
//
// Of a row of n tokens, budget B and R recent ones, a head keeps the R last and the
// B - R older ones of the largest weight.  Kept tokens below B - R stay where they
// are; the others fill the places that fell free there, and the recent ones move to
// [B - R, B): attention does not ask in which order older keys lie (theirs carry
// their positions), so only what has to move moves.
//
// What bounds it: the memory, by the pages' layout.  A moved key is a row, but a moved
// value of a bf16 page two bytes in every 32 of it, so that a page of transposed values
// is read or written nearly whole for one token: 8 prompts of 4096 to 16,384 tokens cut
// to 2048, 4 layers of 8 heads of 128, need 426 MB and move 950 MB (selection 35 us,
// moves 240 us, 4.0 TB/s); 32 rows of 1000 to 1152 tokens, half of them cut, 12 layers
// of 16 heads of 64, need 382 MB, move 670 MB and write most pages in part (44 us and
// 211 us).  The selection is a chain of counts, at most 16, with a barrier each.
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

// Of a unit (layer, row, head): the cache slot that each of its first budget -
// recent places takes its content from, -1 where it keeps its own; and the places
// that take another's as pairs of slots (target, source), one of them -1 if its page
// is not there.
struct EvictWs {
    int32_t* from;                     // [units][stride]
    int2* moves;                       // [units][cap]
    int32_t* count;                    // [units]
    int64_t stride, cap;               // stride: a multiple of 16
};

// Larger weights have larger keys; NaN counts as -infinity.
__device__ __forceinline__ uint32_t key_of(float w) {
    const uint32_t b = __float_as_uint(fmaxf(w, -INFINITY) + 0.f);      // (-0 is 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

struct Unit { int l, c, h, n; };
__device__ __forceinline__ Unit unit_of(const mtp_evict_args& a, int u) {
    Unit x;
    const int H = a.cache.n_kv_heads;
    x.h = u % H;
    x.c = u / H % a.n_rows;
    x.l = u / H / a.n_rows;
    x.n = max(0, min(a.kv_len[x.c], PG * a.max_pages));
    return x;
}

// The counts of the workgroup's set bits before this thread's and in all (buf: NT / 64 ints).
template <int NT>
__device__ __forceinline__ int rank_of(bool set, int& total, int* buf) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t b = __ballot(set);
    __syncthreads();
    if (lane == 0) buf[wave] = __popcll(b);
    __syncthreads();
    int before = 0;
    total = 0;
    for (int i = 0; i < NT / 64; ++i) {
        before += i < wave ? buf[i] : 0;
        total += buf[i];
    }
    return before + __popcll(b & ((1ull << lane) - 1));
}

// The cache slot of token j of row c, -1 in a page outside the pool.
__device__ __forceinline__ int slot_of(const mtp_evict_args& a, const int32_t* tab, int j) {
    const int pg = tab[j / PG];
    return pg >= 0 && pg < a.cache.num_pages ? pg * PG + j % PG : -1;
}

// Which tokens a unit keeps, and their weights.  The bound is the largest key that
// `keep` of the older tokens reach, found two bits at a time by counting: the keys
// stay in registers (E a thread; longer rows are read again each time), and counting
// ends when a bound is reached by exactly `keep`.  Then places and movers are ranked
// in order by ballots.
template <int NT, int E>
__global__ __launch_bounds__(NT) void evict_select_kernel(mtp_evict_args a, EvictWs w) {
    constexpr int NW = NT / 64;
    __shared__ int s_cnt[2][48], s_buf[NW];      // s_cnt: 16 waves of each count
    __shared__ uint32_t s_rank[E * NW];
    __shared__ int s_mover[NT * E / 2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Unit x = unit_of(a, blockIdx.x);
    const bool cut = x.n > a.limit;
    if (x.l == 0 && x.h == 0 && tid == 0) a.out_len[x.c] = cut ? a.budget : x.n;
    const float* in = a.weights + (size_t)blockIdx.x * a.ld;
    float* out = a.out_weights + (size_t)blockIdx.x * a.ld;
    if (!cut) {
        if (out != in)
            for (int j = tid; j < x.n; j += NT) out[j] = in[j];
        return;
    }
    const int keep = a.budget - a.recent, old = x.n - a.recent;
    const int32_t* tab = a.table + (size_t)x.c * a.max_pages;
    int32_t* from = w.from + (size_t)blockIdx.x * w.stride;
    int2* moves = w.moves + (size_t)blockIdx.x * w.cap;
    int holes = 0;
    const bool held = NT < 1024 || old <= NT * E;  // uniform, as all that follows from counts (shorter rows are given to less)
    uint32_t key[E];
    {
        float v[E];
#pragma unroll
        for (int i = 0; i < E; ++i) v[i] = in[min(i * NT + tid, old - 1)];
#pragma unroll
        for (int i = 0; i < E; ++i) key[i] = i * NT + tid < old ? key_of(v[i]) : 0;              // (0: below any weight's)
    }
    uint32_t t = 0;
    int reach = old;                             // tokens whose key is at least t
    for (int bit = 30, buf = 0; bit >= 0 && reach != keep && keep > 0; bit -= 2, buf ^= 1) {
        int n[3] = {0, 0, 0};
        if (held) {
#pragma unroll
            for (int i = 0; i < E; ++i)
#pragma unroll
                for (int k = 0; k < 3; ++k) n[k] += __popcll(__ballot(key[i] >= (t | (uint32_t)(k + 1) << bit)));
        } else {
            for (int j0 = 0; j0 < old; j0 += NT) {
                const uint32_t v = j0 + tid < old ? key_of(in[j0 + tid]) : 0;
#pragma unroll
                for (int k = 0; k < 3; ++k) n[k] += __popcll(__ballot(v >= (t | (uint32_t)(k + 1) << bit)));
            }
        }
        if (lane == 0) {
#pragma unroll
            for (int k = 0; k < 3; ++k) s_cnt[buf][16 * k + wave] = n[k];
        }
        __syncthreads();                         // (the other buffer is read until the next one)
        const uint32_t base = t;
        int part = lane < 48 && lane % 16 < NW ? s_cnt[buf][lane] : 0;
        part += dpp_i<DPP_XOR1>(part);
        part += dpp_i<DPP_XOR2>(part);
        part += dpp_i<DPP_HALF_MIRROR>(part);
        part += dpp_i<DPP_ROR8>(part);
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const int all = __builtin_amdgcn_readlane(part, 16 * k);
            if (all >= keep) {
                t = base | (uint32_t)(k + 1) << bit;
                reach = all;
            }
        }
    }
    if (keep > 0 && held) {
        // of the tokens at the bound the first ones are kept
        int spare = reach - keep;                // tokens at the bound that are not
        uint32_t kept = 0;                       // bit i: key[i] is kept
#pragma unroll
        for (int i = 0; i < E; ++i) kept |= key[i] >= t ? 1u << i : 0;
        if (spare > 0) {                         // (from the last on)
            for (int i = E - 1; i >= 0 && spare > 0; --i) {
                bool at = false;
#pragma unroll
                for (int k = 0; k < E; ++k) at = k == i ? key[k] == t : at;
                int total;
                const int before = rank_of<NT>(at, total, s_buf);
                if (at && before >= total - spare) kept &= ~(1u << i);
                spare -= min(spare, total);
            }
        }
        // places before each wave's of a round, movers (high half) likewise
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int j = i * NT + tid;
            const bool k = kept >> i & 1;
            const uint64_t hole = __ballot(j < keep && !k), mover = __ballot(j >= keep && k);
            if (lane == 0) s_rank[i * NW + wave] = (uint32_t)__popcll(hole) | (uint32_t)__popcll(mover) << 16;
        }
        __syncthreads();
        if (wave == 0) {
            constexpr int PER = (E * NW + 63) / 64;
            uint32_t v[PER], sum = 0;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                v[k] = lane * PER + k < E * NW ? s_rank[lane * PER + k] : 0;
                sum += v[k];
            }
            uint32_t run = sum;
            for (int o = 1; o < 64; o <<= 1) {
                const uint32_t y = __shfl_up(run, o);
                if (lane >= o) run += y;
            }
            run -= sum;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                if (lane * PER + k < E * NW) s_rank[lane * PER + k] = run;
                run += v[k];
            }
            if (lane == 63) s_buf[0] = run & 0xffff;
        }
        __syncthreads();
        const uint64_t lower = (1ull << lane) - 1;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int j = i * NT + tid;
            const bool is = j >= keep && (kept >> i & 1);
            const uint64_t mover = __ballot(is);
            if (is) s_mover[(s_rank[i * NW + wave] >> 16) + __popcll(mover & lower)] = j;
        }
        __syncthreads();
        // (four rounds' loads together; those of places that keep their own token are of that)
#pragma unroll
        for (int i0 = 0; i0 < E; i0 += 4) {
            if (i0 * NT >= keep) break;          // uniform
            int rank[4], page[4], own[4], src[4];
            float v[4];
            bool is[4];
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const int i = i0 + f, j = i * NT + tid;
                is[f] = j < keep && !(kept >> i & 1);
                const uint64_t hole = __ballot(is[f]);
                rank[f] = (s_rank[i * NW + wave] & 0xffff) + __popcll(hole & lower);
                src[f] = is[f] ? s_mover[rank[f]] : min(j, keep - 1);
                page[f] = slot_of(a, tab, src[f]);
                own[f] = slot_of(a, tab, min(j, keep - 1));
                v[f] = in[src[f]];
            }
#pragma unroll
            for (int f = 0; f < 4; ++f) {
                const int j = (i0 + f) * NT + tid;
                if (j >= keep) continue;
                from[j] = is[f] ? page[f] : -1;
                if (is[f]) moves[rank[f]] = make_int2(own[f], page[f]);
                if (is[f] || out != in) out[j] = v[f];
            }
        }
        holes = s_buf[0];
    } else if (keep > 0) {
        int equal_all = 0, total;
        for (int j0 = 0; j0 < old; j0 += NT) {
            rank_of<NT>(j0 + tid < old && key_of(in[j0 + tid]) == t, total, s_buf);
            equal_all += total;
        }
        const int equal_kept = equal_all - (reach - keep);
        for (int pass = 0; pass < 2; ++pass) {   // movers, then the places that they go to
            int equal = 0, done = 0;
            for (int j0 = 0; j0 < (pass ? keep : old); j0 += NT) {
                const int j = j0 + tid;
                const uint32_t k = j < old ? key_of(in[j]) : 0;
                const int e = equal + rank_of<NT>(j < old && k == t, total, s_buf);
                equal += total;
                const bool kept = j < old && (k > t || (k == t && e < equal_kept));
                const bool is = pass ? j < keep && !kept : j >= keep && kept;
                const int at = done + rank_of<NT>(is, total, s_buf);
                done += total;
                holes = done;
                if (pass == 0) {
                    if (is) moves[at].y = j;
                } else if (j < keep) {
                    // (weights move when all of them have been looked at)
                    from[j] = is ? moves[at].y : -1;
                    if (is) moves[at] = make_int2(slot_of(a, tab, j), slot_of(a, tab, moves[at].y));
                }
            }
            __syncthreads();
        }
        for (int j = tid; j < keep; j += NT) {
            const int src = from[j];
            if (src >= 0 || out != in) out[j] = in[src >= 0 ? src : j];
            if (src >= 0) from[j] = slot_of(a, tab, src);
        }
    }
    for (int j = keep + tid; j < ((keep + PG - 1) / PG) * PG; j += NT) from[j] = -1;
    if (tid == 0) w.count[blockIdx.x] = holes;
    // the recent ones' weights, in order: a chunk is read whole before it is written, and writes nothing that a later one reads
    for (int j0 = 0; j0 < a.recent; j0 += NT) {
        const int j = j0 + tid;
        const float v = j < a.recent ? in[old + j] : 0.f;
        __syncthreads();
        if (j < a.recent) out[keep + j] = v;
    }
}

// Moves a unit's keys and values, by a workgroup of NT threads per slice of their
// dimensions: slices share no byte, so that only a workgroup's own steps have to be
// in order (the free places first, then the recent tokens, which overwrite what moved
// there).  Every load of a step is made, from a place that exists, whether its value
// is used or not: loads under a condition were waited for one by one.
typedef uint32_t quad_t __attribute__((ext_vector_type(4)));
// Up to this many tokens move into a page of transposed values on their own, two bytes a dimension; the whole page is read
// and written for more (32 rows of up to 1152 tokens cut to 1024, 1.5 a page: 210 us, 215 us with up to three on their own,
// 235 us with none).
constexpr int FEW = 2;
constexpr int ROW_BYTES = 128;                   // of a token's row that a slice takes
constexpr int TURN_ROWS = 64;                    // dimensions of a transposed block that a slice takes: a lane each
template <typename T, int D>
constexpr int slices() {
    return sizeof(T) == 2 ? D * (int)sizeof(T) / ROW_BYTES + D / TURN_ROWS : 2 * D * (int)sizeof(T) / ROW_BYTES;
}

template <typename T, int D, int NT>
__global__ __launch_bounds__(NT) void evict_move_kernel(mtp_evict_args a, EvictWs w) {
    constexpr int S = slices<T, D>(), KS = D * sizeof(T) / ROW_BYTES;
    const int unit = blockIdx.x / S, slice = blockIdx.x - unit * S, tid = threadIdx.x, lane = tid & 63;
    const Unit x = unit_of(a, unit);
    if (x.n <= a.limit) return;
    const int keep = a.budget - a.recent, H = a.cache.n_kv_heads, old = x.n - a.recent;
    const int32_t* from = w.from + (size_t)unit * w.stride;
    const int32_t* tab = a.table + (size_t)x.c * a.max_pages;
    const size_t blk = (size_t)PG * D, page = 2 * H * blk;
    T* pool = (T*)((char*)a.cache.pool + (size_t)x.l * a.layer_stride) + x.h * blk;
    if (sizeof(T) == 4 || slice < KS) {
        // rows: 16-byte pieces of the slice
        constexpr int PCS = ROW_BYTES / 16, FLY = NT == 1024 ? 4 : 8, TOK = NT / PCS;   // tokens of a step
        T* base = pool + (slice / KS) * H * blk + (slice % KS) * (ROW_BYTES / sizeof(T)) + tid % PCS * (16 / sizeof(T));
        auto at = [&](int slot) { return reinterpret_cast<quad_t*>(base + (size_t)(slot / PG) * page + (slot % PG) * D); };
        const int2* moves = w.moves + (size_t)unit * w.cap;
        const int n = w.count[unit];
        for (int i0 = tid / PCS; i0 < n; i0 += TOK * FLY) {
            int2 m[FLY];
            quad_t v[FLY];
#pragma unroll
            for (int f = 0; f < FLY; ++f) m[f] = moves[min(i0 + TOK * f, n - 1)];
#pragma unroll
            for (int f = 0; f < FLY; ++f) v[f] = *at(max(m[f].y, 0));
#pragma unroll
            for (int f = 0; f < FLY; ++f)
                if (i0 + TOK * f < n && (m[f].x | m[f].y) >= 0) *at(m[f].x) = v[f];
        }
        __syncthreads();
        for (int j0 = tid / PCS; j0 - tid / PCS < a.recent; j0 += TOK * FLY) {
            int src[FLY], dst[FLY];
            quad_t v[FLY];
#pragma unroll
            for (int f = 0; f < FLY; ++f) {
                const int j = min(j0 + TOK * f, a.recent - 1);
                src[f] = slot_of(a, tab, old + j);
                dst[f] = slot_of(a, tab, keep + j);
            }
#pragma unroll
            for (int f = 0; f < FLY; ++f) v[f] = *at(max(src[f], 0));
            __syncthreads();
#pragma unroll
            for (int f = 0; f < FLY; ++f)
                if (j0 + TOK * f < a.recent && (src[f] | dst[f]) >= 0) *at(dst[f]) = v[f];
            __syncthreads();
        }
        return;
    }
    if constexpr (sizeof(T) == 2) {
        // A page a wave: lane l holds eight slots (its half, l % 2) of rows l / 2 and 32 + l / 2, so that a load or store
        // is one contiguous kilobyte.
        constexpr int WAVES = NT / 64;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane & 1;
        T* base = pool + H * blk + (slice - KS) * TURN_ROWS * PG + lane * 8;
        struct Part { quad_t lo, hi; };          // of the two rows
        auto load = [&](int pg) {
            const quad_t* y = reinterpret_cast<const quad_t*>(base + (size_t)pg * page);
            return Part{y[0], y[64]};
        };
        auto store = [&](int pg, const Part& v) {
            quad_t* y = reinterpret_cast<quad_t*>(base + (size_t)pg * page);
            y[0] = v.lo;
            y[64] = v.hi;
        };
        // In LDS a row has 10 words (a column's values, two bytes a lane, then lie in different banks); pieces of 8 bytes.
        constexpr int STR = 20;
        __shared__ __attribute__((aligned(16))) T s_page[WAVES][2][64 * STR];
        T *to = s_page[wave][0], *src = s_page[wave][1];
        auto stage = [&](T* t, const Part& v) {
            uint2* y = reinterpret_cast<uint2*>(t + (lane >> 1) * STR + 8 * half);
            y[0] = make_uint2(v.lo.x, v.lo.y);
            y[1] = make_uint2(v.lo.z, v.lo.w);
            y += 32 * STR / 4;
            y[0] = make_uint2(v.hi.x, v.hi.y);
            y[1] = make_uint2(v.hi.z, v.hi.w);
            __builtin_amdgcn_wave_barrier();
        };
        // The recent ones: each row of the new pages out of two neighbouring old ones, `shift` slots on.  The first ones are
        // asked for before the free places are filled, which changes none of their tokens.
        const int p0 = keep / PG, p1 = max(a.budget - 1, 0) / PG, shift = (old - keep) % PG, ahead = (old - keep) / PG;
        const int last = (x.n - 1) / PG;
        auto page_at = [&](int p) {
            const int pg = __builtin_amdgcn_readfirstlane(tab[min(p, last)]);
            return pg < a.cache.num_pages ? pg : -1;
        };
        int pa = page_at(min(p0 + wave, p1) + ahead), pb = page_at(min(p0 + wave, p1) + ahead + 1);
        Part old_a = load(max(pa, 0)), old_b = load(max(pb, 0));
        for (int p = wave; p * PG < keep; p += WAVES) {
            const int fr = from[p * PG + (lane & (PG - 1))], pg = __builtin_amdgcn_readfirstlane(tab[p]);
            uint32_t holes = (uint32_t)__ballot(fr >= 0) & 0xffffu;
            if (holes == 0 || pg < 0 || pg >= a.cache.num_pages) continue;
            if (__popc(holes) <= FEW) {
                T* row = base - lane * 8 + lane * PG;
                while (holes) {
                    const int k0 = __ffs(holes) - 1;
                    holes &= holes - 1;
                    const int k1 = holes ? __ffs(holes) - 1 : k0;
                    holes &= holes - 1;
                    const int s0 = __builtin_amdgcn_readlane(fr, k0), s1 = __builtin_amdgcn_readlane(fr, k1);
                    const uint32_t v0 = row[(size_t)(s0 / PG) * page + s0 % PG], v1 = row[(size_t)(s1 / PG) * page + s1 % PG];
                    row[(size_t)pg * page + k0] = (T)v0;
                    if (k1 != k0) row[(size_t)pg * page + k1] = (T)v1;
                }
                continue;
            }
            const int mine = fr >= 0 ? fr / PG : -1;                     // lane k: the page that slot k's token comes from
            stage(to, load(pg));
            while (holes) {
                // the next pages that tokens come from, one or three at a time
                const int g0 = __builtin_amdgcn_readlane(mine, __ffs(holes) - 1);
                const uint32_t in0 = (uint32_t)__ballot(mine == g0) & holes;
                auto take = [&](uint32_t in, const Part& y) {
                    if (!in) return;
                    stage(src, y);
                    while (in) {
                        const int k = __ffs(in) - 1, c = __builtin_amdgcn_readlane(fr, k) % PG;
                        in &= in - 1;
                        to[lane * STR + k] = src[lane * STR + c];
                    }
                    __builtin_amdgcn_wave_barrier();
                };
                holes &= ~in0;
                const Part y0 = load(g0);
                if (!holes) {
                    take(in0, y0);
                    break;
                }
                const int g1 = __builtin_amdgcn_readlane(mine, __ffs(holes) - 1);
                const uint32_t in1 = (uint32_t)__ballot(mine == g1) & holes;
                holes &= ~in1;
                const int g2 = holes ? __builtin_amdgcn_readlane(mine, __ffs(holes) - 1) : g1;
                const uint32_t in2 = (uint32_t)__ballot(mine == g2) & holes;
                holes &= ~in2;
                const Part y1 = load(g1), y2 = load(g2);
                take(in0, y0);
                take(in1, y1);
                take(in2, y2);
            }
            Part row;
            const uint2* y = reinterpret_cast<const uint2*>(to + (lane >> 1) * STR + 8 * half);
            const uint2 u0 = y[0], u1 = y[1], u2 = y[32 * STR / 4], u3 = y[32 * STR / 4 + 1];
            row.lo = quad_t{u0.x, u0.y, u1.x, u1.y};
            row.hi = quad_t{u2.x, u2.y, u3.x, u3.y};
            __builtin_amdgcn_wave_barrier();
            store(pg, row);
        }
        __syncthreads();
        if (a.recent == 0) return;
        for (int q = p0; q <= p1; q += WAVES) {
            const int p = q + wave, pg = page_at(min(p, p1));
            // a lane's eight slots come from three neighbouring halves of the old rows: its own and the two behind it, of
            // which another lane has one
            const Part own = load(max(pg, 0));
            uint32_t mask = 0;                   // the slots that a recent token comes to
#pragma unroll
            for (int k = 0; k < PG; ++k) {
                const int j = p * PG + k - keep;
                mask |= j >= 0 && j < a.recent && (k + shift < PG ? pa : pb) >= 0 ? 1u << k : 0;
            }
            const uint32_t here = mask >> 8 * half;
            auto moved = [&](const quad_t& x, const quad_t& y, const quad_t& own) {
                uint32_t r[12];                  // halves h, h + 1 (and a word of h + 2), h = half + shift / 8
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t xo = (uint32_t)dpp_i<DPP_XOR1>((int)x[i]), yo = (uint32_t)dpp_i<DPP_XOR1>((int)y[i]);
                    const uint32_t x0 = half ? xo : x[i], x1 = half ? x[i] : xo, y0 = half ? yo : y[i], y1 = half ? y[i] : yo;
                    const bool next = shift >= 8;
                    r[i] = half ? (next ? y0 : x1) : (next ? x1 : x0);
                    r[4 + i] = half ? (next ? y1 : y0) : (next ? y0 : x1);
                    r[8 + i] = 0;
                }
#pragma unroll
                for (int o = 2; o; o >>= 1)
#pragma unroll
                    for (int i = 0; i + o < 12; ++i) r[i] = shift & 2 * o ? r[i + o] : r[i];
#pragma unroll
                for (int i = 0; i < 4; ++i) r[i] = shift & 1 ? r[i] >> 16 | r[i + 1] << 16 : r[i];
                quad_t z;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t m = (here >> 2 * i & 1 ? 0xffffu : 0) | (here >> (2 * i + 1) & 1 ? 0xffff0000u : 0);
                    z[i] = (r[i] & m) | (own[i] & ~m);
                }
                return z;
            };
            const Part z{moved(old_a.lo, old_b.lo, own.lo), moved(old_a.hi, old_b.hi, own.hi)};
            // (a step's pages lie before all that the next one reads)
            pa = page_at(min(p + WAVES, p1) + ahead);
            pb = page_at(min(p + WAVES, p1) + ahead + 1);
            old_a = load(max(pa, 0));
            old_b = load(max(pb, 0));
            __syncthreads();
            if (p <= p1 && pg >= 0) store(pg, z);
        }
    }
}

bool aligned(const void* p, uintptr_t n) { return p && ((uintptr_t)p & (n - 1)) == 0; }

uint64_t carve(const mtp_evict_args& a, EvictWs* w) {
    const uint64_t units = (uint64_t)a.n_layers * a.n_rows * a.cache.n_kv_heads;
    const int64_t most = (int64_t)PG * a.max_pages, keep = a.budget - a.recent;
    // (a table that cannot hold more than the limit cuts nothing; what moves below budget - recent comes from behind it)
    const int64_t stride = most > a.limit ? (keep + PG - 1) / PG * PG : 0;
    const int64_t cap = most > a.limit ? std::min<int64_t>(keep, most - a.budget) : 0;
    uint64_t o = 0;
    auto take = [&](uint64_t bytes) { uint64_t r = o; o = (o + bytes + 255) & ~uint64_t(255); return r; };
    const uint64_t f = take(units * stride * 4), m = take(units * cap * 8), c = take(units * 4);
    if (w) {
        char* p = (char*)a.workspace;
        w->from = (int32_t*)(p + f); w->moves = (int2*)(p + m); w->count = (int32_t*)(p + c);
        w->stride = stride;
        w->cap = cap;
    }
    return o;
}

int check(const mtp_evict_args* a) {
    if (!a) return MTP_EINVAL;
    const int rc = cache_check(a->cache);
    if (rc != MTP_OK) return rc;
    if (a->n_layers < 1 || a->n_layers > 4096 || a->n_rows < 0 || a->n_rows > 4096 || a->max_pages < 1 || a->max_pages > 65536 ||
        a->recent < 0 || a->budget < a->recent || a->limit < a->budget || a->ld < (int64_t)PG * a->max_pages)
        return MTP_EINVAL;
    // (a launch holds fewer than 2^32 threads: 1024 a unit, or 256 for each of up to eight slices)
    if ((int64_t)a->n_layers * a->n_rows * a->cache.n_kv_heads >= (1ll << 21)) return MTP_EINVAL;
    const uint64_t elt = a->cache.dtype == MTP_DTYPE_BF16 ? 2 : 4;
    const uint64_t layer = (uint64_t)a->cache.num_pages * 2 * a->cache.n_kv_heads * PG * a->cache.head_dim * elt;
    if (a->layer_stride % 16 || (a->n_layers > 1 && a->layer_stride < layer)) return MTP_EINVAL;
    return MTP_OK;
}

// Up to this many slices their workgroups have 1024 threads: long rows move faster with them, the fewer slices the more, short
// ones slower, the more slices the more.  bf16, head dim 128, 4 layers of 8 heads, the whole call with 256 and with 1024
// threads: 512 slices, rows of 2100 to 8000 tokens cut to 2048, 125 and 101 us, of 2300 tokens 50 and 45; 1024 slices, 196 and
// 188, 64 and 73, of 500 to 8192 tokens 183 and 157, of 4096 to 16,384 tokens 294 and 276; 2048 slices 355 and 338, 177 us either
// way, of 1152 tokens with 1000 recent 157 and 182; 4096 slices 627 and 608, 325 and 348, 297 and 354 (the moves alone, 12,288
// slices of rows of up to 1152, half of them cut, 210 and 263 us).  fp32 mostly within
// 5% (up to 6% faster, 12% slower, 4096 slices of 2300 tokens 84 and 105 us).
constexpr unsigned WIDE_GROUPS = 1024;
template <typename T, int D>
int go(hipStream_t st, const mtp_evict_args& a, const EvictWs& w) {
    const unsigned units = (unsigned)(a.n_layers * a.n_rows * a.cache.n_kv_heads);
    const int64_t older = (int64_t)PG * a.max_pages - a.recent;
    // (4 x 8 x 8 rows of 1000 tokens, the whole call: 46.5 us with 256 x 8 keys, 56.1 us with 1024 x 16; 12 x 16 x 16 of 4000:
    // 389 us with 512 x 8, 547 us; 6 x 16 x 16 of 8000: 296 us with 512 x 16, 360 us)
    if (older <= 2048) hipLaunchKernelGGL((evict_select_kernel<256, 8>), dim3(units), dim3(256), 0, st, a, w);
    else if (older <= 4096) hipLaunchKernelGGL((evict_select_kernel<512, 8>), dim3(units), dim3(512), 0, st, a, w);
    else if (older <= 8192) hipLaunchKernelGGL((evict_select_kernel<512, 16>), dim3(units), dim3(512), 0, st, a, w);
    else hipLaunchKernelGGL((evict_select_kernel<1024, 16>), dim3(units), dim3(1024), 0, st, a, w);
    if ((int64_t)PG * a.max_pages > a.limit) {
        if (units * slices<T, D>() <= WIDE_GROUPS)
            hipLaunchKernelGGL((evict_move_kernel<T, D, 1024>), dim3(units * slices<T, D>()), dim3(1024), 0, st, a, w);
        else
            hipLaunchKernelGGL((evict_move_kernel<T, D, 256>), dim3(units * slices<T, D>()), dim3(256), 0, st, a, w);
    }
    return hipGetLastError() == hipSuccess ? MTP_OK : MTP_EHIP;
}

}  // namespace
}  // namespace mtp

extern "C" {

int mtp_pages_evict_workspace_size(const mtp_evict_args* args, uint64_t* bytes) {
    if (mtp::check(args) != MTP_OK || !bytes) return MTP_EINVAL;
    *bytes = args->n_rows == 0 ? 0 : mtp::carve(*args, nullptr);
    return MTP_OK;
}

int mtp_pages_evict(const mtp_evict_args* args, void* hip_stream) {
    using namespace mtp;
    const int rc = check(args);
    if (rc != MTP_OK) return rc;
    const mtp_evict_args& a = *args;
    if (a.n_rows == 0) return MTP_OK;
    if (!aligned(a.table, 4) || !aligned(a.kv_len, 4) || !aligned(a.weights, 4) || !aligned(a.out_weights, 4) ||
        !aligned(a.out_len, 4))
        return MTP_EINVAL;
    EvictWs w{};
    const uint64_t need = carve(a, &w);
    if (need && !aligned(a.workspace, 256)) return MTP_EINVAL;
    if (need > a.workspace_bytes) return MTP_ENOMEM;
    hipStream_t st = (hipStream_t)hip_stream;
    if (a.cache.dtype == MTP_DTYPE_BF16) return a.cache.head_dim == 64 ? go<bf16_t, 64>(st, a, w) : go<bf16_t, 128>(st, a, w);
    return a.cache.head_dim == 64 ? go<float, 64>(st, a, w) : go<float, 128>(st, a, w);
}

}  // extern "C"
