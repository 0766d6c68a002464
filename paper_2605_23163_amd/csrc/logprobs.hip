// Log probability of a given token, entropy and top alternatives of rows of logits.
//
// With m the largest logit of a row, attained first at id a, y_v = (x_v - m) / temperature and
//     S = sum_{v != a} e^y_v,   U = sum_v y_v e^y_v   (the term of a is 0)
// the softmax is p_v = e^y_v / (1 + S), so
//     ln p_v = y_v - ln(1 + S),   entropy = -sum p ln p = ln(1 + S) - U / (1 + S).
// Both terms of the entropy are >= 0, and S without the largest term keeps its digits where the row is nearly certain.
#include <cmath>

#include "fdd_internal.h"
#include "wave.h"

namespace fdd {
namespace {

constexpr int THREADS = 256;
constexpr float LOG2E = 1.4426950408889634f;

struct Args {
    const void* logits;
    const int32_t* tokens;
    const uint8_t* mask;
    float* logprobs;
    float* entropy;
    int32_t* top_ids;
    float* top_logprobs;
    long long V;
    int top;
    float inv_t;
};

// Order of (logit, id): the larger logit first, the lower id among equal ones.  As one unsigned number, larger is earlier.
__device__ __forceinline__ uint64_t key_of(float x, int id)
{
    const uint32_t b = __float_as_uint(x + 0.f);            // (-0 counts as 0)
    const uint32_t u = b & 0x80000000u ? ~b : b | 0x80000000u;
    return ((uint64_t)u << 32) | (uint32_t)~id;
}
__device__ __forceinline__ int key_id(uint64_t k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ float key_logit(uint64_t k)
{
    const uint32_t u = (uint32_t)(k >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}

template <typename T> __device__ __forceinline__ float logit(const T* row, long long v);
template <> __device__ __forceinline__ float logit(const uint16_t* row, long long v) { return __uint_as_float((uint32_t)row[v] << 16); }
template <> __device__ __forceinline__ float logit(const float* row, long long v) { return row[v]; }

template <typename X, typename Op>
__device__ X workgroup_reduce(X x, X* lds, Op op)
{
    const int tid = threadIdx.x;
    lds[tid] = x;
    __syncthreads();
    for (int n = THREADS / 2; n > 0; n /= 2) {
        if (tid < n) lds[tid] = op(lds[tid], lds[tid + n]);
        __syncthreads();
    }
    const X r = lds[0];
    __syncthreads();
    return r;
}

// one workgroup per row
template <typename T>
__global__ __launch_bounds__(THREADS) void logprobs_kernel(Args a)
{
    const size_t r = blockIdx.x;
    if (a.mask && a.mask[r] != 1) return;
    const T* const row = static_cast<const T*>(a.logits) + r * (size_t)a.V;
    const int tid = threadIdx.x;
    __shared__ uint64_t keys[THREADS];
    __shared__ double sums[THREADS];
    auto larger = [](uint64_t p, uint64_t q) { return p > q ? p : q; };
    auto add = [](double p, double q) { return p + q; };

    uint64_t best = 0;
    for (long long v = tid; v < a.V; v += THREADS) best = larger(best, key_of(logit(row, v), (int)v));
    best = workgroup_reduce(best, keys, larger);
    const float m = key_logit(best);
    const int at = key_id(best);

    float s = 0.f, u = 0.f;
    for (long long v = tid; v < a.V; v += THREADS) {
        const float y = fmaxf((logit(row, v) - m) * a.inv_t, -150.f);       // (e^y is 0 from -104 on)
        const float e = v == at ? 0.f : __builtin_amdgcn_exp2f(y * LOG2E);
        s += e;
        u += y * e;
    }
    const double S = workgroup_reduce((double)s, sums, add), U = workgroup_reduce((double)u, sums, add);
    const bool empty = m == -INFINITY;
    const double lse = empty ? (double)NAN : log1p(S);
    if (tid == 0) {
        if (a.logprobs) {
            const int t = a.tokens[r];
            const bool known = t >= 0 && t < a.V;
            a.logprobs[r] = known ? (float)((double)(logit(row, t) - m) * a.inv_t - lse) : -INFINITY;
        }
        if (a.entropy) a.entropy[r] = (float)(lse - U / (1.0 + S));
    }
    if (!a.top_ids) return;
    for (int j = 0; j < a.top; ++j) {
        if (j > 0) {
            const uint64_t last = best;
            best = 0;
            for (long long v = tid; v < a.V; v += THREADS) {
                const uint64_t k = key_of(logit(row, v), (int)v);
                if (k < last) best = larger(best, k);
            }
            best = workgroup_reduce(best, keys, larger);
        }
        if (tid == 0) {
            a.top_ids[r * a.top + j] = key_id(best);
            a.top_logprobs[r * a.top + j] = (float)((double)(key_logit(best) - m) * a.inv_t - lse);
        }
    }
}

}  // namespace

hipError_t launch_logprobs(const fdd_logprob_params& p, hipStream_t s)
{
    Args a;
    a.logits = p.logits;
    a.tokens = p.tokens;
    a.mask = p.row_mask;
    a.logprobs = p.logprobs;
    a.entropy = p.entropy;
    a.top_ids = p.top > 0 ? p.top_ids : nullptr;
    a.top_logprobs = p.top_logprobs;
    a.V = p.V;
    a.top = p.top;
    a.inv_t = 1.f / p.temperature;
    const dim3 grid((unsigned)(p.N * p.B));
    if (p.dtype == FDD_BF16) hipLaunchKernelGGL(logprobs_kernel<uint16_t>, grid, dim3(THREADS), 0, s, a);
    else hipLaunchKernelGGL(logprobs_kernel<float>, grid, dim3(THREADS), 0, s, a);
    return hipGetLastError();
}

}  // namespace fdd

using namespace fdd;

#define fail set_error

static fdd_status check_shape(const fdd_logprob_params* p, const char* fn)
{
    if (!p) return fail(FDD_ERR_NULL, "%s: params is NULL", fn);
    if (p->N <= 0 || p->B <= 0 || p->V <= 0)
        return fail(FDD_ERR_SHAPE, "%s: N, B, V must be positive (got N=%d B=%d V=%lld)", fn, p->N, p->B, (long long)p->V);
    if (p->V >= (1ll << 31)) return fail(FDD_ERR_SHAPE, "%s: V must be below 2^31", fn);
    if ((long long)p->N * p->B > (1ll << 23)) return fail(FDD_ERR_SHAPE, "%s: N*B too large", fn);
    if (p->dtype != FDD_F32 && p->dtype != FDD_BF16) return fail(FDD_ERR_DTYPE, "%s: dtype %d is neither FDD_F32 nor FDD_BF16", fn, p->dtype);
    if (p->top < 0 || p->top > FDD_LOGPROBS_MAX_TOP || p->top > p->V)
        return fail(FDD_ERR_SHAPE, "%s: top=%d outside [0, min(V, %d)]", fn, p->top, FDD_LOGPROBS_MAX_TOP);
    if (p->reserved != 0) return fail(FDD_ERR_UNSUPPORTED, "%s: reserved field must be 0", fn);
    return FDD_OK;
}

extern "C" {

size_t fdd_token_logprobs_workspace(const fdd_logprob_params* p)
{
    if (check_shape(p, "fdd_token_logprobs_workspace") != FDD_OK) return 0;
    return 0;
}

fdd_status fdd_token_logprobs(const fdd_logprob_params* p)
{
    const char* const fn = "fdd_token_logprobs";
    fdd_status st = check_shape(p, fn);
    if (st != FDD_OK) return st;
    if (!(p->temperature > 0.f) || std::isinf(p->temperature) || std::isinf(1.f / p->temperature))
        return fail(FDD_ERR_UNSUPPORTED, "%s: temperature must be positive and finite, and so must its reciprocal", fn);
    if (!p->logits) return fail(FDD_ERR_NULL, "%s: logits must not be NULL", fn);
    if (p->logprobs && !p->tokens) return fail(FDD_ERR_NULL, "%s: logprobs need tokens", fn);
    if (p->top > 0 && !p->top_ids != !p->top_logprobs) return fail(FDD_ERR_NULL, "%s: top_ids and top_logprobs come together", fn);
    if (!p->logprobs && !p->entropy && !(p->top > 0 && p->top_ids)) return fail(FDD_ERR_NULL, "%s: no output to compute", fn);
    if (reinterpret_cast<uintptr_t>(p->logits) & 15u) return fail(FDD_ERR_UNSUPPORTED, "%s: logits must be 16-byte aligned", fn);
    const void* words[] = {p->tokens, p->logprobs, p->entropy, p->top_ids, p->top_logprobs};
    for (const void* w : words)
        if (reinterpret_cast<uintptr_t>(w) & 3u) return fail(FDD_ERR_UNSUPPORTED, "%s: tokens and outputs must be 4-byte aligned", fn);
    hipError_t e = launch_logprobs(*p, static_cast<hipStream_t>(p->stream));
    if (e != hipSuccess) return fail(FDD_ERR_LAUNCH, "%s: launch failed: %s", fn, hipGetErrorString(e));
    return FDD_OK;
}

}  // extern "C"
