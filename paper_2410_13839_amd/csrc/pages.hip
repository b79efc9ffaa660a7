// Paged serving: block tables and slot maps from lengths (mtp_pages_plan),
// cache writes (mtp_pages_write) and page copies (mtp_pages_copy).
//
// The plan keeps no free list: a page is free when no row of the new tables
// keeps it, so the tables themselves are the allocator's state.  Three steps:
// every row's lengths, fresh pages and running sums (one workgroup); every row
// marks the pages that it keeps in a bitmap; every row takes its fresh pages by
// rank among the clear bits and writes its table row, slots and positions.
// In all but the largest plans every row's workgroup finds out by itself what
// the others keep, so that the three steps are one launch.
// What bounds it: the chain of dependent loads (parent -> lengths -> table ->
// marks) and the launches, not bytes: 8 rows of 229 pages 6.2 us, 256 beams of
// 256 pages 13.5 us, 256 rows of 512 15.8 us in three launches.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/mtp.h"
#include "common.h"

namespace mtp {
namespace {

constexpr int PG = 16;                 // tokens per page
constexpr int MAX_ROWS = 4096;
constexpr int ROWS_T = 1024;           // threads of the step that takes every row
constexpr int PLAN_T = 256;            // threads of the other two
// One launch up to these sizes: table entries, pages (a byte of LDS each) and
// rows (a workgroup each, so one or two a CU).  64 rows of 64 pages 7.4 us instead
// of 11.3 us in three launches, 256 of 256 (beams) 13.5 and 14.8 us, 256 of 512
// 20.6 and 15.8 us.  Workgroups of 256 threads, whose sums are shorter, for few
// pieces of 64 entries: 8 rows of 229 pages 6.2 us, 7.8 us with 1024 threads; 256
// rows of 16 pages 14.7 and 10.2 us.
constexpr int ONE_ENTRIES = 1 << 16, ONE_PAGES = 1 << 17, ONE_ROWS = 256, FEW_PIECES = 64;

// Row c of the plan: its parent, the parent's cached tokens, its new tokens
// (the sign bit: its partly filled last page becomes a fresh one), and the
// fresh pages of the rows before it.
typedef int4 PlanRow;
__device__ __forceinline__ int row_new(const PlanRow& r) { return r.z & 0x7fffffff; }
__device__ __forceinline__ bool row_moved(const PlanRow& r) { return r.z < 0; }
__device__ __forceinline__ int row_kept(const PlanRow& r) { return r.y / PG + (r.y % PG > 0 && !row_moved(r) ? 1 : 0); }
__device__ __forceinline__ int row_need(const PlanRow& r) { return (r.y + row_new(r) + PG - 1) / PG; }

struct PlanWs {
    uint32_t* bits;                    // [words] pages kept
    PlanRow* rows;                     // [n_rows]
};

uint64_t plan_words(int num_pages) { return ((uint64_t)num_pages + 31) / 32; }

bool plan_is_one(const mtp_plan_args& a) {
    return a.n_rows <= ONE_ROWS && a.num_pages <= ONE_PAGES && (int64_t)a.n_rows * a.max_pages <= ONE_ENTRIES;
}

uint64_t plan_carve(const mtp_plan_args& a, PlanWs* w) {
    if (plan_is_one(a)) return 0;
    uint64_t o = 0;
    auto take = [&](uint64_t bytes) { uint64_t r = o; o = (o + bytes + 255) & ~uint64_t(255); return r; };
    const uint64_t b = take(plan_words(a.num_pages) * 4), f = take((uint64_t)a.n_rows * 16);
    if (w) {
        char* p = (char*)a.workspace;
        w->bits = (uint32_t*)(p + b); w->rows = (PlanRow*)(p + f);
    }
    return o;
}

// Exclusive sums over the workgroup's NT threads; v becomes the sum of the
// threads before, the result is the total.  buf: NT / 64 values of LDS.
template <int NT, typename T>
__device__ __forceinline__ T block_scan(T& v, T* buf) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const T own = v;
    T x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const T y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();                   // (buf may still be read from the last call)
    if (lane == 63) buf[wave] = x;
    __syncthreads();
    T before = 0, total = 0;
    for (int i = 0; i < NT / 64; ++i) {
        before += i < wave ? buf[i] : 0;
        total += buf[i];
    }
    v = before + x - own;
    return total;
}

// Step 1 by one workgroup of NT threads: r[k], row tid + NT k (empty behind the
// last), and with `lead` row_start and kv_len; start: r[PER - 1]'s first token.
// low: n_rows words of LDS.  The totals' low half counts fresh pages, the high
// half new tokens (fewer than 2^31: the table holds fewer than 2^27 pages);
// bad: this thread's rows outside their range.
template <int NT, int PER>
__device__ __forceinline__ uint64_t plan_rows(const mtp_plan_args& a, PlanRow (&r)[PER], int* low, uint64_t* buf,
                                              uint64_t& start, bool lead, int& bad) {
    const int tid = threadIdx.x, n = a.n_rows;
    for (int c = tid; c < n; c += NT) low[c] = 0x7fffffff;
    __syncthreads();
    bad = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int c = tid + NT * k;
        r[k] = make_int4(0, 0, 0, 0);
        if (c >= n) continue;
        int p = a.parent ? a.parent[c] : c;
        const int A = a.add[c];
        bool ok = p >= 0 && p < n && A >= 0;
        if (!ok) p = 0;
        const int L = a.len[p];
        ok = ok && L >= 0 && (int64_t)L + A <= (int64_t)PG * a.max_pages;
        if (ok) {
            r[k] = make_int4(p, L, A, 0);
            if (a.parent) atomicMin(&low[p], c);
        }
        bad += ok ? 0 : 1;
    }
    __syncthreads();
    uint64_t sum = 0;                  // of the slabs before
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        if (NT * k >= n) break;        // uniform
        const int c = tid + NT * k;
        const bool in = c < n;
        if (in && a.parent && r[k].y % PG && low[r[k].x] != c) r[k].z |= (int)0x80000000;
        uint64_t v = in ? (uint64_t)row_new(r[k]) << 32 | (uint32_t)(row_need(r[k]) - row_kept(r[k])) : 0;
        const uint64_t all = block_scan<NT>(v, buf);
        r[k].w = (int)(uint32_t)(sum + v);
        start = (sum + v) >> 32;
        if (in && lead) {
            a.row_start[c] = (int)start;
            a.kv_len[c] = r[k].y + row_new(r[k]);
        }
        sum += all;
    }
    if (lead && tid == 0) a.row_start[n] = (int)(sum >> 32);
    return sum;
}

// Step 2 for row r by `nt` threads (this one is `i`).
__device__ __forceinline__ void plan_mark(const mtp_plan_args& a, const PlanRow& r, uint32_t* bits, int i, int nt) {
    const int keep = row_kept(r);
    const int32_t* src = a.table_in + (size_t)r.x * a.max_pages;
    int bad = 0;
    for (int j = i; j < keep; j += nt) {
        const int pg = src[j];
        if (pg >= 0 && pg < a.num_pages) atomicOr(&bits[pg >> 5], 1u << (pg & 31));
        else ++bad;
    }
    if (bad) atomicAdd(&a.status[2], bad);
}

// The clear bits of word i (pages that nobody keeps).
__device__ __forceinline__ uint32_t free_bits(const uint32_t* bits, int i, int num_pages) {
    const uint32_t b = ~bits[i];
    const int left = num_pages - 32 * i;
    return left < 32 ? b & ((1u << left) - 1) : b;
}

// Free pages before each thread's run of `per` words, into before[0 .. NT].
template <int NT>
__device__ __forceinline__ void plan_count(const uint32_t* bits, int num_pages, int per, int* before, int* buf) {
    const int words = (num_pages + 31) / 32, w0 = min((int)threadIdx.x * per, words), w1 = min(w0 + per, words);
    int cnt = 0;
    for (int i = w0; i < w1; ++i) cnt += __popc(free_bits(bits, i, num_pages));
    const int all = block_scan<NT>(cnt, buf);
    before[threadIdx.x] = cnt;
    if (threadIdx.x == 0) before[NT] = all;
    __syncthreads();
}

// The run that holds the free page of rank k < before[NT]; k becomes its rank there.
template <int NT>
__device__ __forceinline__ int plan_run(const int* before, int& k) {
    int lo = 0, hi = NT;               // before[lo] <= k < before[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (before[mid] <= k) lo = mid; else hi = mid;
    }
    k -= before[lo];
    return lo;
}

// The page of rank k among the free ones, -1 past the last.
template <int NT>
__device__ __forceinline__ int plan_page(const uint32_t* bits, int num_pages, int per, const int* before, int k) {
    if (k >= before[NT]) return -1;
    int i = plan_run<NT>(before, k) * per;
    uint32_t b = free_bits(bits, i, num_pages);
    while (k >= __popc(b)) {
        k -= __popc(b);
        b = free_bits(bits, ++i, num_pages);
    }
    for (; k > 0; --k) b &= b - 1;
    return i * 32 + __ffs(b) - 1;
}

// Step 3's table row by `nt` threads, page(k) the free page of rank k; the
// caller synchronises before plan_slots.  The result: pages that there were not.
template <typename F>
__device__ __forceinline__ int plan_table(const mtp_plan_args& a, int c, const PlanRow& r, int i, int nt, F page) {
    const int keep = row_kept(r), need = row_need(r);
    const int32_t* src = a.table_in + (size_t)r.x * a.max_pages;
    int32_t* dst = a.table + (size_t)c * a.max_pages;
    int missing = 0;
    for (int j = i; j < a.max_pages; j += nt) {
        int pg = -1;
        if (j < keep) {
            pg = src[j];
            if (pg < 0 || pg >= a.num_pages) pg = -1;
        } else if (j < need) {
            pg = page(r.w + (j - keep));
            missing += pg < 0 ? 1 : 0;
        }
        dst[j] = pg;
    }
    return missing;
}

// Slots, positions and the page copy of row c, its table row written.
__device__ __forceinline__ void plan_slots(const mtp_plan_args& a, int c, const PlanRow& r, int64_t t0, int i, int nt) {
    const int32_t* dst = a.table + (size_t)c * a.max_pages;
    for (int k = i; k < row_new(r) && t0 + k < a.max_tokens; k += nt) {
        const int pos = r.y + k, pg = dst[pos / PG];
        a.slots[t0 + k] = pg >= 0 ? pg * PG + pos % PG : -1;
        a.positions[t0 + k] = pos;
    }
    if (i == 0) {
        int s = -1, d = -1;
        if (row_moved(r)) {
            s = a.table_in[(size_t)r.x * a.max_pages + r.y / PG];
            d = dst[r.y / PG];
            if (s < 0 || s >= a.num_pages || d < 0) s = d = -1;
        }
        a.copies[2 * c] = s;
        a.copies[2 * c + 1] = d;
    }
}

// -1 behind the last token.
__device__ __forceinline__ void plan_rest(const mtp_plan_args& a, int64_t tokens, int64_t i, int64_t nt) {
    for (int64_t t = tokens + i; t < a.max_tokens; t += nt) {
        a.slots[t] = -1;
        a.positions[t] = -1;
    }
}

__device__ __forceinline__ int tokens_lost(const mtp_plan_args& a, uint64_t sum) {
    return (int)max((int64_t)(sum >> 32) - a.max_tokens, (int64_t)0);
}

__global__ __launch_bounds__(ROWS_T) void plan_rows_kernel(mtp_plan_args a, PlanWs w) {
    __shared__ int s_low[MAX_ROWS];
    __shared__ uint64_t s_buf[ROWS_T / 64];
    if (blockIdx.x == 0) {
        constexpr int PER = MAX_ROWS / ROWS_T;
        PlanRow r[PER];
        int bad;
        uint64_t start;
        const uint64_t sum = plan_rows<ROWS_T, PER>(a, r, s_low, s_buf, start, true, bad);
#pragma unroll
        for (int k = 0; k < PER; ++k)
            if ((int)threadIdx.x + ROWS_T * k < a.n_rows) w.rows[threadIdx.x + ROWS_T * k] = r[k];
        uint64_t b = bad;
        const uint64_t all_bad = block_scan<ROWS_T>(b, s_buf);
        if (threadIdx.x == 0) {
            a.status[0] = 0;
            a.status[1] = (int)all_bad;
            a.status[2] = 0;
            a.status[3] = tokens_lost(a, sum);
        }
        return;
    }
    const int words = (a.num_pages + 31) / 32;
    for (int i = (blockIdx.x - 1) * ROWS_T + threadIdx.x; i < words; i += (gridDim.x - 1) * ROWS_T) w.bits[i] = 0u;
}

__global__ __launch_bounds__(PLAN_T) void plan_mark_kernel(mtp_plan_args a, PlanWs w) {
    plan_mark(a, w.rows[blockIdx.x], w.bits, threadIdx.x, PLAN_T);
}

__global__ __launch_bounds__(PLAN_T) void plan_assign_kernel(mtp_plan_args a, PlanWs w, int per) {
    __shared__ int s_before[PLAN_T + 1], s_buf[PLAN_T / 64];
    const int c = blockIdx.x;
    const PlanRow r = w.rows[c];
    if (row_need(r) > row_kept(r)) plan_count<PLAN_T>(w.bits, a.num_pages, per, s_before, s_buf);
    const int missing = plan_table(a, c, r, threadIdx.x, PLAN_T,
                                   [&](int k) { return plan_page<PLAN_T>(w.bits, a.num_pages, per, s_before, k); });
    if (missing) atomicAdd(&a.status[0], missing);
    __syncthreads();
    plan_slots(a, c, r, a.row_start[c], threadIdx.x, PLAN_T);
    plan_rest(a, a.row_start[a.n_rows], (int64_t)c * PLAN_T + threadIdx.x, (int64_t)gridDim.x * PLAN_T);
}

// Free pages among the 16 of a quad, and the page of rank k among those of the
// quads from i on (there is one).
__device__ __forceinline__ int quad_free(const uint4& x) {
    return 16 - __popc(x.x) - __popc(x.y) - __popc(x.z) - __popc(x.w);
}
__device__ __forceinline__ int free_byte(const uint4* used, int i, int k) {
    uint4 x = used[i];
    for (int f = quad_free(x); k >= f; f = quad_free(x)) {
        k -= f;
        x = used[++i];
    }
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t b = ~w[0] & 0x01010101u;
    int at = 0;
#pragma unroll
    for (int q = 1; q < 4; ++q)
        if (k >= __popc(b)) {
            k -= __popc(b);
            b = ~w[q] & 0x01010101u;
            at = 4 * q;
        }
    for (; k > 0; --k) b &= b - 1;
    return 16 * i + at + ((__ffs(b) - 1) >> 3);
}

// All three steps by a workgroup per row: each takes every row's lengths and,
// where its own row (or the status, workgroup 0's) needs to know the free
// pages, marks what every row keeps in LDS, a byte a page (stores without
// atomics: neighbouring pages, which a row mostly has, would queue up at the
// words of a bitmap).
template <int NT, bool BEAMS>
__global__ __launch_bounds__(NT) void plan_alone_kernel(mtp_plan_args a) {
    constexpr int FLY = 4;             // pieces in flight per wave
    __shared__ uint4 s_used[ONE_PAGES / 16];
    // up to 64 kept entries of a row: the first in table_in; their number, with BEAMS also bit 7, the last is a partly
    // filled page, and from bit 8 on how many rows keep the others
    __shared__ int2 s_piece[ONE_ENTRIES / 64 + ONE_ROWS];
    __shared__ PlanRow s_own;
    __shared__ int s_low[ONE_ROWS], s_keep[ONE_ROWS], s_buf[NT / 64], s_before[NT + 1], s_start, s_bad[2];
    __shared__ uint64_t s_sum[NT / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = blockIdx.x;
    const bool lead = c == 0;
    const int quads = (a.num_pages + 15) / 16, per = (quads + NT - 1) / NT;
    if (tid < 2) s_bad[tid] = 0;
    if (BEAMS && tid < ONE_ROWS) s_keep[tid] = 0;
    int bad;
    uint64_t start;
    PlanRow mine[1];
    const uint64_t sum = plan_rows<NT, 1>(a, mine, s_low, s_sum, start, lead, bad);
    if (lead && bad) atomicAdd(&s_bad[0], bad);
    if (tid == c) { s_own = mine[0]; s_start = (int)start; }
    // of the rows that continue one parent the lowest keeps all that any of them does and marks it (256 beams of 256 pages
    // 14.8 us if all of them do)
    const bool in = tid < a.n_rows && mine[0].y > 0;
    if (BEAMS && in) atomicAdd(&s_keep[mine[0].x], 1);
    const int kept = in && (!BEAMS || s_low[mine[0].x] == tid) ? row_kept(mine[0]) : 0;
    int at = (kept + 63) / 64;
    const int pieces = block_scan<NT>(at, s_buf);
    const PlanRow r = s_own;
    const bool fresh = lead || row_need(r) > row_kept(r);      // uniform
    if (fresh) {
        const int keepers = BEAMS && kept > 0 ? s_keep[mine[0].x] << 8 : 0, part = BEAMS && kept > mine[0].y / PG ? 128 : 0;
        for (int j = 0; j < kept; j += 64)
            s_piece[at++] = make_int2(mine[0].x * a.max_pages + j, min(kept - j, 64) | keepers | (j + 64 >= kept ? part : 0));
        for (int i = tid; i < quads; i += NT) s_used[i] = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
        uint8_t* used = reinterpret_cast<uint8_t*>(s_used);
        bad = 0;
        for (int u0 = wave; u0 < pieces; u0 += NT / 64 * FLY) {
            int pg[FLY], n[FLY];
#pragma unroll
            for (int k = 0; k < FLY; ++k) {
                const int u = u0 + NT / 64 * k;
                const int2 x = s_piece[min(u, pieces - 1)];
                n[k] = u < pieces ? x.y : 0;
                pg[k] = lane < (BEAMS ? n[k] & 127 : n[k]) ? a.table_in[x.x + lane] : -1;
            }
#pragma unroll
            for (int k = 0; k < FLY; ++k) {
                if ((uint32_t)pg[k] < (uint32_t)a.num_pages) used[pg[k]] = 1;
                else if (BEAMS) bad += lane >= (n[k] & 127) ? 0 : (n[k] & 128) && lane == (n[k] & 127) - 1 ? 1 : n[k] >> 8;
                else bad += lane < n[k] ? 1 : 0;
            }
        }
        if (lead && bad) atomicAdd(&s_bad[1], bad);
        if (tid < quads * 16 - a.num_pages) used[a.num_pages + tid] = 1;
        __syncthreads();
        const int q0 = min(tid * per, quads), q1 = min(q0 + per, quads);
        int cnt = 0;
        for (int i = q0; i < q1; ++i) cnt += quad_free(s_used[i]);
        const int all = block_scan<NT>(cnt, s_buf);
        s_before[tid] = cnt;
        if (tid == 0) s_before[NT] = all;
        __syncthreads();
    }
    if (lead && tid == 0) {
        a.status[0] = max((int)(uint32_t)sum - s_before[NT], 0);
        a.status[1] = s_bad[0];
        a.status[2] = s_bad[1];
        a.status[3] = tokens_lost(a, sum);
    }
    plan_table(a, c, r, tid, NT, [&](int k) {
        if (k >= s_before[NT]) return -1;
        return free_byte(s_used, plan_run<NT>(s_before, k) * per, k);
    });
    __syncthreads();
    plan_slots(a, c, r, s_start, tid, NT);
    plan_rest(a, sum >> 32, (int64_t)c * NT + tid, (int64_t)gridDim.x * NT);
}

bool aligned(const void* p, uintptr_t n) { return p && ((uintptr_t)p & (n - 1)) == 0; }

int plan_check(const mtp_plan_args* a) {
    if (!a) return MTP_EINVAL;
    if (a->n_rows < 0 || a->n_rows > MAX_ROWS || a->max_pages < 1 || a->max_pages > 65536 || a->num_pages < 1 ||
        a->num_pages >= (1 << 27) || a->max_tokens < 0 || (int64_t)a->n_rows * a->max_pages >= (1 << 27))
        return MTP_EINVAL;
    return MTP_OK;
}

// ------------------------------------------------------------------ writes
//
// One workgroup per (group of tokens, KV head).  Keys and fp32 values are rows
// of the page: 16-byte pieces.  A bf16 page's V block is transposed: the
// group's values pass through LDS, and eight tokens in a row that go to eight
// slots in a row from a multiple of eight on (an octet) are stored as one
// 16-byte piece per dimension; other tokens store two bytes a dimension.  An
// octet belongs to its first token's group, which also loads the up to seven
// tokens behind its own; every group looks at 7 + 48 + 7 slots, a lane each, so
// that all agree on the octets wherever the groups' borders fall.
// What bounds it: HBM.  32 prompts of 200 to 450 tokens, 16 heads of 64 in bf16
// (85 MB read and written): 18 us warm, 25 us from HBM (3.4 TB/s; groups of 16
// tokens without the look around, 31 us: octets across their borders were
// stored in two-byte pieces), fp32 37 us (4.6 TB/s).
constexpr int WOWN = 48, WEXT = 7;     // a group's own tokens, tokens looked at on either side

template <typename T, int D>
__global__ __launch_bounds__(256) void pages_write_kernel(mtp_write_args a) {
    constexpr int PER = 16 / sizeof(T), PCS = D / PER;          // elements of a piece, pieces of a row
    constexpr int STR = D + 8;                                  // padded LDS row
    constexpr bool TURN = sizeof(T) == 2;
    __shared__ __attribute__((aligned(16))) T s_v[TURN ? (WOWN + WEXT) * STR : 1];
    __shared__ int s_slot[64], s_oct[WOWN / 8];
    const int H = a.cache.n_kv_heads, h = blockIdx.x % H, t0 = blockIdx.x / H * WOWN, tid = threadIdx.x, lane = tid & 63;
    const int lim = a.cache.num_pages * PG;
    // lane i: token t0 - 7 + i (every wave looks for itself)
    const int64_t tl = (int64_t)t0 - WEXT + lane;
    int slot = lane < WOWN + 2 * WEXT && tl >= 0 && tl < a.n_tokens ? a.slots[tl] : -1;
    if (slot < 0 || slot >= lim) slot = -1;
    if (tid < 64) s_slot[tid] = slot;
    uint64_t heads = 0, alone = 0;     // bit i, lane i's token: the first of an octet; in none
    if constexpr (TURN) {
        const int next = __shfl_down(slot, 1);
        const uint64_t follows = __ballot(lane < 63 && slot >= 0 && next == slot + 1);
        heads = __ballot(slot >= 0 && slot % 8 == 0 && lane <= 63 - 8 && ((follows >> lane) & 0x7f) == 0x7f);
        uint64_t covered = heads | heads << 1;
        covered |= covered << 2;
        covered |= covered << 4;
        constexpr uint64_t OWN = ((1ull << WOWN) - 1) << WEXT;
        alone = __ballot(slot >= 0) & ~covered & OWN;
        heads &= OWN;
        if (tid < 64 && (heads >> lane & 1)) s_oct[__popcll(heads & ((1ull << lane) - 1))] = lane;
    }
    __syncthreads();
    T* pool = (T*)a.cache.pool;
    const size_t blk = (size_t)PG * D;
    for (int i = tid; i < (TURN ? WOWN + WEXT : WOWN) * PCS; i += 256) {
        const int tok = i / PCS, pc = i % PCS, s = s_slot[WEXT + tok];
        if (s < 0) continue;
        const int64_t t = t0 + tok;
        T* page = pool + (size_t)(s / PG) * 2 * H * blk;
        if (tok < WOWN)
            *reinterpret_cast<uint4*>(page + h * blk + (s % PG) * D + pc * PER) =
                *reinterpret_cast<const uint4*>((const T*)a.k + t * a.k_stride + h * D + pc * PER);
        const uint4 vv = *reinterpret_cast<const uint4*>((const T*)a.v + t * a.v_stride + h * D + pc * PER);
        if constexpr (TURN) *reinterpret_cast<uint4*>(&s_v[tok * STR + pc * PER]) = vv;
        else *reinterpret_cast<uint4*>(page + (H + h) * blk + (s % PG) * D + pc * PER) = vv;
    }
    if constexpr (TURN) {
        __syncthreads();
        // octets in pairs, whose 16-byte pieces alternate: those of one page make 32 bytes in a row per dimension
        const int n = __popcll(heads);
        for (int i = tid; i < (n + 1) / 2 * 2 * D; i += 256) {
            const int o = i / (2 * D) * 2 + (i & 1), d = (i % (2 * D)) >> 1;
            if (o >= n) continue;
            const int at = s_oct[o], s = s_slot[at];
            const T* row = &s_v[(at - WEXT) * STR + d];
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = (uint32_t)row[2 * j * STR] | (uint32_t)row[(2 * j + 1) * STR] << 16;
            *reinterpret_cast<uint4*>(pool + (size_t)(s / PG) * 2 * H * blk + (H + h) * blk + s % PG + d * PG) =
                make_uint4(w[0], w[1], w[2], w[3]);
        }
        if (alone == 0) return;                                 // uniform
        for (int i = tid; i < WOWN * D; i += 256) {
            const int tok = i / D, d = i % D;
            if (!(alone >> (WEXT + tok) & 1)) continue;
            const int s = s_slot[WEXT + tok];
            pool[(size_t)(s / PG) * 2 * H * blk + (H + h) * blk + d * PG + s % PG] = s_v[tok * STR + d];
        }
    }
}

template <typename T, int D>
void write_go(hipStream_t st, const mtp_write_args& a) {
    const unsigned groups = (unsigned)((a.n_tokens + WOWN - 1) / WOWN);
    hipLaunchKernelGGL((pages_write_kernel<T, D>), dim3(groups * a.cache.n_kv_heads), dim3(256), 0, st, a);
}

// ------------------------------------------------------------------ copies
//
// One workgroup per (copy, layer), 16 bytes a thread and step, up to 1024
// threads as the page has pieces.  Bound by HBM: 0.6 x 256 pages of 64 KB in 12
// layers (242 MB read and written) 43 us warm, 55 us from HBM (4.4 TB/s; 59 us
// with 256 threads, 79 us with those and eight loads of a thread in flight; 52
// us with loads and stores that pass the caches by, which 32 copies, 24 MB, pay
// for: 11.4 us instead of 9.5).
__global__ __launch_bounds__(1024) void pages_copy_kernel(mtp_copy_args a) {
    const int i = blockIdx.x;
    const int src = a.copies[2 * i], dst = a.copies[2 * i + 1];
    if (src < 0 || src >= a.num_pages || dst < 0 || dst >= a.num_pages || src == dst) return;
    for (int l = blockIdx.y; l < a.n_layers; l += gridDim.y) {
        char* base = (char*)a.pool + (size_t)l * a.layer_stride;
        const uint4* s = (const uint4*)(base + (size_t)src * a.page_bytes);
        uint4* d = (uint4*)(base + (size_t)dst * a.page_bytes);
        for (uint64_t k = threadIdx.x; k < a.page_bytes / 16; k += blockDim.x) d[k] = s[k];
    }
}

int launched() { return hipGetLastError() == hipSuccess ? MTP_OK : MTP_EHIP; }

}  // namespace

// Whether a cache description is usable; shared with the attention.
int cache_check(const mtp_cache& c) {
    if (!aligned(c.pool, 16)) return MTP_EINVAL;
    if (c.dtype != MTP_DTYPE_F32 && c.dtype != MTP_DTYPE_BF16) return MTP_EINVAL;
    if (c.num_pages < 1 || c.num_pages >= (1 << 27)) return MTP_EINVAL;
    if (c.n_kv_heads < 1 || c.n_kv_heads > 1024) return MTP_EINVAL;
    if (c.head_dim != 64 && c.head_dim != 128) return MTP_EINVAL;
    return MTP_OK;
}

}  // namespace mtp

extern "C" {

int mtp_pages_plan_workspace_size(const mtp_plan_args* args, uint64_t* bytes) {
    const int rc = mtp::plan_check(args);
    if (rc != MTP_OK || !bytes) return MTP_EINVAL;
    *bytes = mtp::plan_carve(*args, nullptr);
    return MTP_OK;
}

int mtp_pages_plan(const mtp_plan_args* args, void* hip_stream) {
    using namespace mtp;
    const int rc = plan_check(args);
    if (rc != MTP_OK) return rc;
    const mtp_plan_args& a = *args;
    if (a.n_rows == 0) return MTP_OK;
    if ((a.parent && !aligned(a.parent, 4)) || !aligned(a.len, 4) || !aligned(a.add, 4) || !aligned(a.table_in, 4) ||
        !aligned(a.table, 4) || !aligned(a.row_start, 4) || !aligned(a.kv_len, 4) || !aligned(a.copies, 4) ||
        !aligned(a.status, 4))
        return MTP_EINVAL;
    if (a.max_tokens > 0 && (!aligned(a.slots, 4) || !aligned(a.positions, 4))) return MTP_EINVAL;
    if (a.parent && a.table == a.table_in) return MTP_EINVAL;
    PlanWs w{};
    const uint64_t need = plan_carve(a, &w);
    if (need && !aligned(a.workspace, 256)) return MTP_EINVAL;
    if (need > a.workspace_bytes) return MTP_ENOMEM;
    hipStream_t st = (hipStream_t)hip_stream;
    const int words = (int)plan_words(a.num_pages);
    if (need == 0) {
        if (a.n_rows * ((a.max_pages + 63) / 64) <= FEW_PIECES) {
            if (a.parent) hipLaunchKernelGGL((plan_alone_kernel<256, true>), dim3(a.n_rows), dim3(256), 0, st, a);
            else hipLaunchKernelGGL((plan_alone_kernel<256, false>), dim3(a.n_rows), dim3(256), 0, st, a);
        } else {
            if (a.parent) hipLaunchKernelGGL((plan_alone_kernel<1024, true>), dim3(a.n_rows), dim3(1024), 0, st, a);
            else hipLaunchKernelGGL((plan_alone_kernel<1024, false>), dim3(a.n_rows), dim3(1024), 0, st, a);
        }
        return launched();
    }
    const int cb = (words + ROWS_T * 4 - 1) / (ROWS_T * 4);
    hipLaunchKernelGGL(plan_rows_kernel, dim3(1 + (cb < 256 ? cb : 256)), dim3(ROWS_T), 0, st, a, w);
    hipLaunchKernelGGL(plan_mark_kernel, dim3(a.n_rows), dim3(PLAN_T), 0, st, a, w);
    hipLaunchKernelGGL(plan_assign_kernel, dim3(a.n_rows), dim3(PLAN_T), 0, st, a, w, (words + PLAN_T - 1) / PLAN_T);
    return launched();
}

int mtp_pages_write(const mtp_write_args* args, void* hip_stream) {
    using namespace mtp;
    if (!args || args->n_tokens < 0) return MTP_EINVAL;
    const mtp_write_args& a = *args;
    const int rc = cache_check(a.cache);
    if (rc != MTP_OK) return rc;
    if (a.n_tokens == 0) return MTP_OK;
    const int64_t row = (int64_t)a.cache.n_kv_heads * a.cache.head_dim, per = a.cache.dtype == MTP_DTYPE_BF16 ? 8 : 4;
    if (!aligned(a.slots, 4) || !aligned(a.k, 16) || !aligned(a.v, 16) || a.k_stride < row || a.v_stride < row ||
        a.k_stride % per || a.v_stride % per)
        return MTP_EINVAL;
    hipStream_t st = (hipStream_t)hip_stream;
    // (a launch holds fewer than 2^32 threads)
    if (((int64_t)a.n_tokens + WOWN - 1) / WOWN * a.cache.n_kv_heads >= (1ll << 24)) return MTP_EINVAL;
    if (a.cache.dtype == MTP_DTYPE_BF16) a.cache.head_dim == 64 ? write_go<bf16_t, 64>(st, a) : write_go<bf16_t, 128>(st, a);
    else a.cache.head_dim == 64 ? write_go<float, 64>(st, a) : write_go<float, 128>(st, a);
    return launched();
}

int mtp_pages_copy(const mtp_copy_args* args, void* hip_stream) {
    using namespace mtp;
    if (!args) return MTP_EINVAL;
    const mtp_copy_args& a = *args;
    if (a.n_copies < 0 || a.n_copies > MAX_ROWS || a.n_layers < 0 || a.n_layers > 4096 || a.num_pages < 1 ||
        a.num_pages >= (1 << 27) || a.page_bytes == 0 || a.page_bytes % 16 || a.layer_stride % 16 ||
        a.page_bytes > (1u << 30))
        return MTP_EINVAL;
    if (a.n_layers > 1 && a.layer_stride < (uint64_t)a.num_pages * a.page_bytes) return MTP_EINVAL;
    if (a.n_copies == 0 || a.n_layers == 0) return MTP_OK;
    if (!aligned(a.pool, 16) || !aligned(a.copies, 4)) return MTP_EINVAL;
    const uint64_t pieces = a.page_bytes / 16;
    const unsigned threads = pieces >= 1024 ? 1024 : (unsigned)(pieces + 63) / 64 * 64;
    hipLaunchKernelGGL(pages_copy_kernel, dim3(a.n_copies, a.n_layers), dim3(threads), 0, (hipStream_t)hip_stream, a);
    return launched();
}

}  // extern "C"
