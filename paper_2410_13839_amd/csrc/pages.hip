// Paged serving: block tables and slot maps from lengths (mtp_pages_plan),
// cache writes (mtp_pages_write) and page copies (mtp_pages_copy).
//
// The plan keeps no free list: a page is free when no row of the new tables
// keeps it, so the tables themselves are the allocator's state.  Three
// launches: clear the page bitmap; every row marks the pages that it keeps and
// stores how many fresh ones it wants; every row takes its fresh pages by rank
// among the clear bits and writes its table row, slots and positions.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/mtp.h"
#include "common.h"

namespace mtp {
namespace {

constexpr int PG = 16;                 // tokens per page
constexpr int PLAN_T = 256;            // threads of the plan's workgroups
constexpr int MAX_ROWS = 4096;

struct PlanWs {
    uint32_t* bits;                    // [words] pages kept
    int32_t* fresh;                    // [n_rows] fresh pages a row wants
    int32_t* adds;                     // [n_rows] its new tokens (0 for a bad row)
};

uint64_t plan_words(int num_pages) { return ((uint64_t)num_pages + 31) / 32; }

uint64_t plan_carve(const mtp_plan_args& a, PlanWs* w) {
    uint64_t o = 0;
    auto take = [&](uint64_t bytes) { uint64_t r = o; o = (o + bytes + 255) & ~uint64_t(255); return r; };
    const uint64_t b = take(plan_words(a.num_pages) * 4), f = take((uint64_t)a.n_rows * 4), d = take((uint64_t)a.n_rows * 4);
    if (w) {
        char* p = (char*)a.workspace;
        w->bits = (uint32_t*)(p + b); w->fresh = (int32_t*)(p + f); w->adds = (int32_t*)(p + d);
    }
    return o;
}

// What row c continues; L and A are 0 for a bad row (ok false).
struct PlanRow { int p, L, A; bool ok; };
__device__ __forceinline__ PlanRow plan_row(const mtp_plan_args& a, int c) {
    PlanRow r;
    r.p = a.parent ? a.parent[c] : c;
    r.A = a.add[c];
    r.ok = r.p >= 0 && r.p < a.n_rows && r.A >= 0;
    r.L = r.ok ? a.len[r.p] : 0;
    r.ok = r.ok && r.L >= 0 && (int64_t)r.L + r.A <= (int64_t)PG * a.max_pages;
    if (!r.ok) { r.p = 0; r.L = 0; r.A = 0; }
    return r;
}

__global__ __launch_bounds__(PLAN_T) void plan_clear_kernel(mtp_plan_args a, PlanWs w) {
    const uint64_t n = ((uint64_t)a.num_pages + 31) / 32;
    for (uint64_t i = (uint64_t)blockIdx.x * PLAN_T + threadIdx.x; i < n; i += (uint64_t)gridDim.x * PLAN_T) w.bits[i] = 0u;
    if (blockIdx.x == 0 && threadIdx.x < 4) a.status[threadIdx.x] = 0;
}

// Whether an earlier row continues p too (uniform; every thread calls it).
__device__ __forceinline__ bool plan_follows(const mtp_plan_args& a, int c, int p) {
    int hit = 0;
    if (a.parent)
        for (int i = threadIdx.x; i < c; i += PLAN_T) {
            const PlanRow r = plan_row(a, i);
            hit |= (r.ok && r.p == p) ? 1 : 0;
        }
    return __syncthreads_or(hit) != 0;
}

__global__ __launch_bounds__(PLAN_T) void plan_mark_kernel(mtp_plan_args a, PlanWs w) {
    const int c = blockIdx.x;
    const PlanRow r = plan_row(a, c);
    const int full = r.L / PG, part = r.L % PG > 0, need = (r.L + r.A + PG - 1) / PG;
    const bool follows = part && r.ok && plan_follows(a, c, r.p);
    const int keep = full + (part && !follows ? 1 : 0);
    const int32_t* src = a.table_in + (size_t)r.p * a.max_pages;
    int bad = 0;
    for (int j = threadIdx.x; j < keep; j += PLAN_T) {
        const int pg = src[j];
        if (pg >= 0 && pg < a.num_pages) atomicOr(&w.bits[pg >> 5], 1u << (pg & 31));
        else ++bad;
    }
    if (bad) atomicAdd(&a.status[2], bad);
    if (threadIdx.x == 0) {
        w.fresh[c] = need - keep;
        // (the sign bit tells the next launch that the row's last page moved)
        w.adds[c] = r.A | (follows ? (int)0x80000000 : 0);
        a.kv_len[c] = r.L + r.A;
        if (!r.ok) atomicAdd(&a.status[1], 1);
    }
}

__device__ __forceinline__ int64_t wave_sum64_i(int64_t v) {
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

__global__ __launch_bounds__(PLAN_T) void plan_assign_kernel(mtp_plan_args a, PlanWs w) {
    __shared__ int64_t s_f[PLAN_T / 64], s_a[PLAN_T / 64], s_t[PLAN_T / 64];
    __shared__ int32_t s_free[PLAN_T + 1];       // free pages before each thread's run of words
    const int c = blockIdx.x, tid = threadIdx.x;
    // fresh pages and new tokens of the rows before c, and all new tokens
    int64_t nf = 0, na = 0, nt = 0;
    for (int i = tid; i < a.n_rows; i += PLAN_T) {
        const int ad = w.adds[i] & 0x7fffffff;
        if (i < c) { nf += w.fresh[i]; na += ad; }
        nt += ad;
    }
    nf = wave_sum64_i(nf); na = wave_sum64_i(na); nt = wave_sum64_i(nt);
    if ((tid & 63) == 0) { s_f[tid >> 6] = nf; s_a[tid >> 6] = na; s_t[tid >> 6] = nt; }
    // free pages: each thread counts a run of bitmap words
    const int words = (a.num_pages + 31) / 32, per = (words + PLAN_T - 1) / PLAN_T;
    const int w0 = min(tid * per, words), w1 = min(w0 + per, words);
    auto free_bits = [&](int i) {
        const uint32_t b = ~w.bits[i];
        return i == words - 1 && (a.num_pages & 31) ? b & ((1u << (a.num_pages & 31)) - 1) : b;
    };
    const int want = w.fresh[c];
    int cnt = 0;
    if (want > 0)
        for (int i = w0; i < w1; ++i) cnt += __popc(free_bits(i));
    s_free[tid + 1] = cnt;
    if (tid == 0) s_free[0] = 0;
    __syncthreads();
    for (int o = 1; o < PLAN_T; o <<= 1) {
        const int v = tid + 1 > o ? s_free[tid + 1 - o] : 0;
        __syncthreads();
        s_free[tid + 1] += v;
        __syncthreads();
    }
    nf = na = nt = 0;
    for (int i = 0; i < PLAN_T / 64; ++i) { nf += s_f[i]; na += s_a[i]; nt += s_t[i]; }

    const PlanRow r = plan_row(a, c);
    const int total = r.L + r.A, full = r.L / PG, part = r.L % PG > 0, need = (total + PG - 1) / PG;
    const bool moved = w.adds[c] < 0;
    const int keep = need - want;
    const int32_t* src = a.table_in + (size_t)r.p * a.max_pages;
    int32_t* dst = a.table + (size_t)c * a.max_pages;
    int missing = 0;
    for (int j = tid; j < a.max_pages; j += PLAN_T) {
        int pg = -1;
        if (j < keep) {
            pg = src[j];
            if (pg < 0 || pg >= a.num_pages) pg = -1;
        } else if (j < need) {
            // the page of rank nf + j - keep among the free ones
            const int64_t k64 = nf + (j - keep);
            if (k64 >= s_free[PLAN_T]) {
                ++missing;
            } else {
                int k = (int)k64, lo = 0, hi = PLAN_T;      // s_free[lo] <= k < s_free[hi]
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (s_free[mid] <= k) lo = mid; else hi = mid;
                }
                k -= s_free[lo];
                int i = min(lo * per, words);
                uint32_t b = free_bits(i);
                while (k >= __popc(b)) { k -= __popc(b); b = free_bits(++i); }
                for (; k > 0; --k) b &= b - 1;
                pg = i * 32 + __ffs(b) - 1;
            }
        }
        dst[j] = pg;
    }
    if (missing) atomicAdd(&a.status[0], missing);
    __syncthreads();
    // slots and positions of the row's tokens
    int lost = 0;
    for (int i = tid; i < r.A; i += PLAN_T) {
        const int64_t t = na + i;
        if (t >= a.max_tokens) { ++lost; continue; }
        const int pos = r.L + i, pg = dst[pos / PG];
        a.slots[t] = pg >= 0 ? pg * PG + pos % PG : -1;
        a.positions[t] = pos;
    }
    if (lost) atomicAdd(&a.status[3], lost);
    // entries behind the last token
    for (int64_t t = nt + (int64_t)c * PLAN_T + tid; t < a.max_tokens; t += (int64_t)gridDim.x * PLAN_T) {
        a.slots[t] = -1;
        a.positions[t] = -1;
    }
    if (tid == 0) {
        a.row_start[c] = (int32_t)(na < 0x7fffffff ? na : 0x7fffffff);
        if (c == a.n_rows - 1) a.row_start[a.n_rows] = (int32_t)(nt < 0x7fffffff ? nt : 0x7fffffff);
        int s = -1, d = -1;
        if (moved && part) {
            s = src[full];
            if (s < 0 || s >= a.num_pages) s = -1;
            d = dst[full];
            if (s < 0 || d < 0) s = d = -1;
        }
        a.copies[2 * c] = s;
        a.copies[2 * c + 1] = d;
    }
}

bool aligned(const void* p, uintptr_t n) { return p && ((uintptr_t)p & (n - 1)) == 0; }

int plan_check(const mtp_plan_args* a) {
    if (!a) return MTP_EINVAL;
    if (a->n_rows < 0 || a->n_rows > MAX_ROWS || a->max_pages < 1 || a->max_pages > 65536 || a->num_pages < 1 ||
        a->num_pages >= (1 << 27) || a->max_tokens < 0)
        return MTP_EINVAL;
    return MTP_OK;
}

// ------------------------------------------------------------------ writes
template <typename T>
__global__ __launch_bounds__(256) void pages_write_kernel(mtp_write_args a) {
    const int D = a.cache.head_dim, H = a.cache.n_kv_heads;
    const int t = blockIdx.x;
    const int slot = a.slots[t];
    if (slot < 0 || slot >= a.cache.num_pages * PG) return;
    T* page = (T*)a.cache.pool + (size_t)(slot / PG) * 2 * H * PG * D;
    const T* k = (const T*)a.k + (int64_t)t * a.k_stride;
    const T* v = (const T*)a.v + (int64_t)t * a.v_stride;
    const int s = slot % PG;
    for (int i = threadIdx.x; i < H * D; i += 256) {
        const int h = i / D, d = i % D;
        page[(size_t)h * PG * D + s * D + d] = k[i];
        page[(size_t)(H + h) * PG * D + (sizeof(T) == 2 ? d * PG + s : s * D + d)] = v[i];
    }
}

// ------------------------------------------------------------------ copies
__global__ __launch_bounds__(256) void pages_copy_kernel(mtp_copy_args a) {
    const int i = blockIdx.x;
    const int src = a.copies[2 * i], dst = a.copies[2 * i + 1];
    if (src < 0 || src >= a.num_pages || dst < 0 || dst >= a.num_pages || src == dst) return;
    for (int l = blockIdx.y; l < a.n_layers; l += gridDim.y) {
        char* base = (char*)a.pool + (size_t)l * a.layer_stride;
        const uint4* s = (const uint4*)(base + (size_t)src * a.page_bytes);
        uint4* d = (uint4*)(base + (size_t)dst * a.page_bytes);
        for (uint64_t k = threadIdx.x; k < a.page_bytes / 16; k += 256) d[k] = s[k];
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
        !aligned(a.status, 4) || !aligned(a.workspace, 256))
        return MTP_EINVAL;
    if (a.max_tokens > 0 && (!aligned(a.slots, 4) || !aligned(a.positions, 4))) return MTP_EINVAL;
    if (a.parent && a.table == a.table_in) return MTP_EINVAL;
    PlanWs w{};
    if (plan_carve(a, &w) > a.workspace_bytes) return MTP_ENOMEM;
    hipStream_t st = (hipStream_t)hip_stream;
    const uint64_t words = plan_words(a.num_pages);
    const unsigned cb = (unsigned)((words + PLAN_T * 4 - 1) / (PLAN_T * 4));
    hipLaunchKernelGGL(plan_clear_kernel, dim3(cb < 1024 ? cb : 1024), dim3(PLAN_T), 0, st, a, w);
    hipLaunchKernelGGL(plan_mark_kernel, dim3(a.n_rows), dim3(PLAN_T), 0, st, a, w);
    hipLaunchKernelGGL(plan_assign_kernel, dim3(a.n_rows), dim3(PLAN_T), 0, st, a, w);
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
    if (a.cache.dtype == MTP_DTYPE_BF16)
        hipLaunchKernelGGL((pages_write_kernel<uint16_t>), dim3(a.n_tokens), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((pages_write_kernel<float>), dim3(a.n_tokens), dim3(256), 0, st, a);
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
    hipLaunchKernelGGL(pages_copy_kernel, dim3(a.n_copies, a.n_layers), dim3(256), 0, (hipStream_t)hip_stream, a);
    return launched();
}

}  // extern "C"
