// Reductions over a wavefront, shared by the kernels that end in one.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fdd {

// Reductions over the 64 lanes, result in every lane: DPP moves within rows of 16 (pairs, quads, then mirrors, which
// pair up what the steps before have made uniform), gfx950 lane swaps across rows.  A shuffle through LDS takes 60
// cycles and more per step, and a workgroup of the vocabulary pass ended with 18 of them in six dependent steps (pass
// with sums 41.0 -> 39.1 us, without 36.6 -> 34.1 at N=16, B=64, V=152064; 16.5 -> 15.6 and 13.9 -> 13.0 at N=8, B=32).
template <typename Op>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t x, Op op)
{
    x = op(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true));    // quad_perm 1 0 3 2
    x = op(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true));    // quad_perm 2 3 0 1
    x = op(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xF, 0xF, true));   // row_half_mirror
    x = op(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xF, 0xF, true));   // row_mirror
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = op(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return op(b[0], b[1]);
}

}  // namespace fdd
