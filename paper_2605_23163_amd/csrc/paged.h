// What the operators on a paged cache and on trees of drafted tokens share.
#pragma once
#include <cmath>

#include "fdd_internal.h"

namespace fdd {

inline bool aligned_to(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool spans_overlap(const void* p, unsigned long long n, const void* q, unsigned long long m)
{
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return n > 0 && m > 0 && a < b + m && b < a + n;
}
// Whether one of the outputs overlaps an input or another output (arrays that are not there have no bytes)
struct Span {
    const void* p;
    unsigned long long bytes;
};
template <int OUTS, int INS>
bool outputs_overlap(const Span (&outs)[OUTS], const Span (&ins)[INS])
{
    for (int i = 0; i < OUTS; ++i) {
        for (int j = 0; j < INS; ++j)
            if (outs[i].p && ins[j].p && spans_overlap(outs[i].p, outs[i].bytes, ins[j].p, ins[j].bytes)) return true;
        for (int j = 0; j < i; ++j)
            if (outs[i].p && outs[j].p && spans_overlap(outs[i].p, outs[i].bytes, outs[j].p, outs[j].bytes)) return true;
    }
    return false;
}
// (by its bits: some files are compiled without NaN)
inline bool finite_bits(float x) { return ((__builtin_bit_cast(uint32_t, x) >> 23) & 255u) != 255u; }
inline long long dtype_bytes(int dtype) { return dtype == FDD_BF16 ? 2 : 4; }

// The cache's own fields; bytes of one of its two pools.
fdd_status check_paged_cache(const fdd_paged_cache* c, const char* fn);
inline unsigned long long pool_bytes(const fdd_paged_cache& c)
{
    return (unsigned long long)c.pages * c.page_size * c.Hkv * c.D * dtype_bytes(c.dtype);
}
// A stride of tokens (0 = dense): at least a token, 16-byte aligned
fdd_status check_token_stride(long long stride, long long token, int dtype, const char* what, const char* fn);
inline long long token_stride(long long stride, long long token) { return stride ? stride : token; }

// The parent of token i of a tree, or -1: `given` is its entry.
__host__ __device__ __forceinline__ int parent_of(int i, int given) { return given >= 0 && given < i ? given : -1; }

}  // namespace fdd
