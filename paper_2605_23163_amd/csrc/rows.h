// Which row of logits a workgroup takes where only some rows are to be read: shared by the vocabulary passes.
#pragma once
#include "fdd_internal.h"

namespace fdd {

// Which (row, piece) a workgroup of a vocabulary pass takes: workgroup u the piece u mod vsplits of the (u / vsplits)-th
// ELIGIBLE row, so that the live workgroups come first and together, and the dispatcher deals them out evenly.  (With
// row = u / vsplits, workgroups of rows that are not eligible left at once, but not before they had been dealt a place:
// a scaffold pattern, which all rollouts share, left some compute units with several live workgroups and others with
// none.)  Every wavefront counts for itself: a lane looks at 16 positions, ballots give the counts before it, no LDS and no
// barrier; mask and scaffold are read in one round trip.  Returns -1 past the last eligible row.  Up to LIVE_ROWS rows, which a
// wavefront reads at once; `deal_to_eligible` has the calls it pays for, the others go by `unit_of_workgroup` below.
constexpr int LIVE_ROWS = 1024;
__device__ __forceinline__ int eligible_row(const uint8_t* mask, const uint8_t* scaffold, int rows, int target)
{
    const int lane = thread_id_x() & 63;
    const int at = lane * 16, p = min(at, rows - 16), drop = at - p;         // (drop: positions the lanes below have already)
    const uint8_t* const sc = scaffold ? scaffold : mask;
    const uint32_t use_sc = scaffold ? ~0u : 0u;
    uint32_t m[4], s[4];
    __builtin_memcpy(m, mask + p, 16);    // (positions start anywhere: the loads need no alignment)
    __builtin_memcpy(s, sc + p, 16);
    uint32_t z[4];                        // 0x80 in the bytes of eligible positions
    int c = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint32_t t = (m[w] ^ 0x01010101u) | (s[w] & use_sc);                    // zero bytes: mask 1, no scaffold
        const uint32_t e = ~(((t & 0x7f7f7f7fu) + 0x7f7f7f7fu) | t | 0x7f7f7f7fu);
        z[w] = drop >= 4 * w + 4 ? 0u : drop <= 4 * w ? e : e & (~0u << (8 * (drop - 4 * w)));
        c += __builtin_popcount(z[w]);
    }
    int before = 0;                       // eligible positions of the lanes below
#pragma unroll
    for (int b = 0; b < 5; ++b) {
        const uint64_t has = __builtin_amdgcn_ballot_w64((c >> b) & 1);
        before += (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(has >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)has, 0u)) << b;
    }
    const uint64_t here = __builtin_amdgcn_ballot_w64(before <= target && target < before + c);
    if (here == 0) return -1;
    const int l = __builtin_ctzll(here);
    int left = target - __builtin_amdgcn_readlane(before, l);
    const int first = __builtin_amdgcn_readlane(p, l);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t e = (uint32_t)__builtin_amdgcn_readlane((int)z[w], l);
        const int n = __builtin_popcount(e);
        if (left < n) {
            for (; left > 0; --left) e &= e - 1;
            return first + 4 * w + (__builtin_ctz(e) >> 3);
        }
        left -= n;
    }
    return -1;
}

// Other calls: each group of 8 consecutive launch indices (workgroups are dealt to the 8 XCDs round-robin) is
// rotated, by an amount that changes from group to group, from 8 groups to the next 8 and from 64 to the next, so that a
// scaffold pattern that repeats from rollout to rollout does not load the XCDs unequally.
__device__ __forceinline__ unsigned unit_of_workgroup(unsigned n_units)
{
    const unsigned u = wg_id_x(), g = u >> 3;
    if ((g << 3) + 8u > n_units) return u;           // a last, incomplete group stays as it is
    return (g << 3) + ((u + g + (g >> 3) + (g >> 6) + (g >> 9)) & 7u);
}

}  // namespace fdd
