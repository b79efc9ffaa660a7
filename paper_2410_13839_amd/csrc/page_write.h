// What the kernels that write tokens into cache pages share: a group of tokens
// of one KV head, whose slots every wave looks up, and the transposed V blocks
// of bf16 pages.
//
// Keys and fp32 values are rows of the page.  A bf16 page's V block is
// transposed: the group's values pass through LDS, and eight tokens in a row
// that go to eight slots in a row from a multiple of eight on (an octet) are
// stored as one 16-byte piece per dimension; other tokens store two bytes a
// dimension.  An octet belongs to its first token's group, which also loads the
// up to seven tokens behind its own; every group looks at 7 + 48 + 7 slots (of few tokens at 7 + 8 + 7), a
// lane each, so that all agree on the octets wherever the groups' borders fall.
#pragma once

#include "common.h"

namespace mtp {

constexpr int PAGE_TOK = 16;           // tokens per page
constexpr int WOWN = 48, WEXT = 7;     // a group's own tokens, tokens looked at on either side

// Bit i, lane i's token: the first of an octet; in none.
struct WriteOctets { uint64_t heads, alone; };

// The slots of the group of tokens t0 .. t0 + WOWN - 1 into s_slot (entry i: token t0 -
// 7 + i; -1 where there is none), and with TURN its octets, whose entries go to
// s_oct.  slot_of(t): the slot of token t, by the caller's own rule.  The caller
// synchronises.
template <bool TURN, int WOWN = mtp::WOWN, typename F>
__device__ __forceinline__ WriteOctets write_find(int t0, int n_tokens, int lim, int* s_slot, int* s_oct, F slot_of) {
    const int tid = threadIdx.x, lane = tid & 63;
    // lane i: token t0 - 7 + i (every wave looks for itself)
    const int64_t tl = (int64_t)t0 - WEXT + lane;
    int slot = lane < WOWN + 2 * WEXT && tl >= 0 && tl < n_tokens ? slot_of(tl) : -1;
    if (slot < 0 || slot >= lim) slot = -1;
    if (tid < 64) s_slot[tid] = slot;
    uint64_t heads = 0, alone = 0;
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
    return WriteOctets{heads, alone};
}

// The group's values, rows of D + 8 elements in s_v from token t0 on, into the
// transposed V blocks of head h, by 256 threads.
template <typename T, int D, int WOWN = mtp::WOWN>
__device__ __forceinline__ void write_turned(T* pool, int H, int h, const WriteOctets& oct, const int* s_slot, const int* s_oct,
                                             const T* s_v) {
    constexpr int STR = D + 8;
    const size_t blk = (size_t)PAGE_TOK * D;
    const int tid = threadIdx.x;
    // octets in pairs, whose 16-byte pieces alternate: those of one page make 32 bytes in a row per dimension
    const int n = __popcll(oct.heads);
    for (int i = tid; i < (n + 1) / 2 * 2 * D; i += 256) {
        const int o = i / (2 * D) * 2 + (i & 1), d = (i % (2 * D)) >> 1;
        if (o >= n) continue;
        const int at = s_oct[o], s = s_slot[at];
        const T* row = &s_v[(at - WEXT) * STR + d];
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = (uint32_t)row[2 * j * STR] | (uint32_t)row[(2 * j + 1) * STR] << 16;
        *reinterpret_cast<uint4*>(pool + (size_t)(s / PAGE_TOK) * 2 * H * blk + (H + h) * blk + s % PAGE_TOK + d * PAGE_TOK) =
            make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (oct.alone == 0) return;                                 // uniform
    for (int i = tid; i < WOWN * D; i += 256) {
        const int tok = i / D, d = i % D;
        if (!(oct.alone >> (WEXT + tok) & 1)) continue;
        const int s = s_slot[WEXT + tok];
        pool[(size_t)(s / PAGE_TOK) * 2 * H * blk + (H + h) * blk + d * PAGE_TOK + s % PAGE_TOK] = s_v[tok * STR + d];
    }
}

}  // namespace mtp
