// The prefix cache in 8 bits: rows are quantised as they join it, and read back.
//
// With s = 2^e the scale of a block of 64 rows of a head, e = min{ e : max |x| <= 448 * 2^e } and -117 <= e <= 119,
//     code = e4m3(x / s),  value = code * s.
// max |x| = m 2^E with 1 <= m < 2, so e = E - 8 if m <= 1.75 and E - 7 if not: the scale comes from the bits of the
// largest magnitude, and dividing by it is exact.  Powers of two cost a floating-point code nothing but up to one
// binade of the range below its smallest normal number, and they make everything after the one rounding exact: a
// value has four significant bits, so it is a bf16 number (2^-9 * 2^-117 is the smallest bf16 normal one), codes can
// move to a larger scale, and attention multiplies the values that are read back here.
//
// Both kernels are bound by the bytes that they move, short calls by their launch (32 rows 2.5 and 1.9 us).  Written and read back, arrays in
// rotation so that all of it comes from memory, a launch included: 32768 rows of 8 x 128 bf16 40 and 42 us (5.0 and 4.8 TB/s read and
// written), 16384 of 4 x 128 14.3 and 12.4 (3.5 and 4.1), fp32 18.8 and 17.6 (4.5 and 4.8).  The 84 MB of the second fit the last-level cache: the
// same arrays again and again take 12.9 and 11.5.
// A thread takes as many elements at a time as 16 bytes of the rows hold (8
// bf16, 4 fp32), so that neighbouring lanes load or store neighbouring pieces.
//   quantize    one workgroup per (block of 64 rows, KV head, K or V): it holds the block in registers between the
//               maximum and the rounding, so a row is read once.
//   dequantize  threads in the order of the destination.
#include <cmath>
#include <cstdlib>
#include <type_traits>

#include "fdd_internal.h"
#include "wave.h"

namespace fdd {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int QB = FDD_QUANT_BLOCK;
constexpr int THREADS = 256;

// one of K and V
struct Side {
    void* rows;                 // source or destination
    long long row_stride;       // elements
    uint8_t* codes;
    float* scale;
};

struct QuantArgs {
    Side side[2];
    int Hkv, capacity, row0, rows;
};

struct DequantArgs {
    Side side[2];
    int Hkv, capacity, row0, rows;
    FastDiv dHkv;
    long long code_bs, scale_bs, rows_bs;    // batch: elements from one problem to the next
};

// 16 bytes of rows as fp32 and back
__device__ __forceinline__ void widen(const u32x4& w, float (&x)[8])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(w[j] << 16);
        x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
}
__device__ __forceinline__ void widen(const u32x4& w, float (&x)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = __uint_as_float(w[j]);
}
__device__ __forceinline__ u32x4 narrow(const float (&x)[8])
{
    u32x4 w;
    // (four significant bits: the upper half of the word is the value)
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (__float_as_uint(x[2 * j]) >> 16) | (__float_as_uint(x[2 * j + 1]) & 0xffff0000u);
    return w;
}
__device__ __forceinline__ u32x4 narrow(const float (&x)[4])
{
    return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}

// the codes that belong to them
template <int VEC>
struct Codes {
    uint32_t w[VEC / 4];
};
template <int VEC>
__device__ __forceinline__ Codes<VEC> load_codes(const uint8_t* p)
{
    Codes<VEC> c;
    __builtin_memcpy(&c, __builtin_assume_aligned(p, VEC), VEC);
    return c;
}
template <int VEC>
__device__ __forceinline__ void store_codes(uint8_t* p, const Codes<VEC>& c)
{
    __builtin_memcpy(__builtin_assume_aligned(p, VEC), &c, VEC);
}

template <int VEC>
__device__ __forceinline__ void decode(const Codes<VEC>& c, float scale, float (&x)[VEC])
{
#pragma unroll
    for (int i = 0; i < VEC / 4; ++i) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.w[i], true);
        x[4 * i] = lo[0] * scale;
        x[4 * i + 1] = lo[1] * scale;
        x[4 * i + 2] = hi[0] * scale;
        x[4 * i + 3] = hi[1] * scale;
    }
}

template <int VEC>
__device__ __forceinline__ Codes<VEC> encode(const float (&x)[VEC], float inv)
{
    float y[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const float t = x[i] * inv;
        y[i] = t != t ? t : fminf(fmaxf(t, -448.f), 448.f);     // (the conversion makes NaN of what is too large)
    }
    Codes<VEC> c;
#pragma unroll
    for (int i = 0; i < VEC / 4; ++i) {
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
        c.w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], w, true);
    }
    return c;
}

// grid (blocks of the cache that the rows touch, Hkv, K and V)
template <int D, typename T>
__global__ __launch_bounds__(THREADS, 6) void quantize_kernel(QuantArgs a)
{
    constexpr int VEC = 16 / sizeof(T);
    constexpr int CPR = D / VEC;                      // pieces of a row
    constexpr int ROWS = THREADS / CPR, NC = QB / ROWS;   // rows a step; steps: pieces of a thread
    const Side& s = a.side[blockIdx.z];
    const int h = blockIdx.y, tid = threadIdx.x, block = a.row0 / QB + (int)blockIdx.x;
    const int lead = max(a.row0 - block * QB, 0);     // rows of the block that are there already
    const int end = min(a.row0 + a.rows - block * QB, QB);
    uint8_t* const codes = s.codes + ((size_t)h * a.capacity + (size_t)block * QB) * D;
    float* const scale_at = s.scale + (size_t)h * (a.capacity / QB) + block;

    const float old = lead > 0 ? *scale_at : 0.f;
    const int r0 = tid / CPR, col = tid % CPR;
    const T* const src = static_cast<const T*>(s.rows) + ((long long)block * QB - a.row0 + r0) * s.row_stride + h * D + col * VEC;   // (used from row `lead` on)
    u32x4 raw[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int r = r0 + c * ROWS;
        raw[c] = u32x4{0u, 0u, 0u, 0u};
        if (r >= lead && r < end) raw[c] = *reinterpret_cast<const u32x4*>(src + c * ROWS * s.row_stride);
    }
    uint32_t top = 0;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        float x[VEC];
        widen(raw[c], x);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const uint32_t b = __float_as_uint(x[j]) & 0x7fffffffu;
            top = max(top, b < 0x7f800000u ? b : 0u);
        }
    }
    __shared__ uint32_t part[THREADS / 64];
    top = wave_reduce(top, [](uint32_t p, uint32_t q) { return max(p, q); });
    if ((tid & 63) == 0) part[tid >> 6] = top;
    __syncthreads();
    top = max(max(part[0], part[1]), max(part[2], part[3]));
    int e = (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = min(max(e, -117), 119);
    const float scale = fmaxf(__uint_as_float((uint32_t)(e + 127) << 23), old), inv = 1.f / scale;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int r = r0 + c * ROWS;
        float x[VEC];
        widen(raw[c], x);
        if (r >= lead && r < end) store_codes<VEC>(codes + (size_t)(tid + c * THREADS) * VEC, encode<VEC>(x, inv));
    }
    if (lead > 0 && scale != old) {
#pragma unroll 1
        for (int r = r0; r < lead; r += ROWS) {
            uint8_t* const at = codes + r * D + col * VEC;
            float x[VEC];
            decode<VEC>(load_codes<VEC>(at), old, x);
            store_codes<VEC>(at, encode<VEC>(x, inv));
        }
    }
    if (tid == 0) *scale_at = scale;
}

// grid (pieces / (THREADS PIECES), K and V, problems); a thread's pieces are all requested before the first is stored.  us with 1, 2, 4
// of them: 16384 rows of 4 x 128 fp32 19.2, 17.6, 18.5, bf16 12.6, 12.4, 12.6; 8000 7.3, 6.8, 7.0; 32 1.9, 2.0, 2.5; 32768 of 8 x 128
// bf16 40.0, 42.1, 43.9.
constexpr int PIECES = 2;
template <int D, typename T>
__global__ __launch_bounds__(THREADS) void dequantize_kernel(DequantArgs a)
{
    constexpr int VEC = 16 / sizeof(T), CPR = D / VEC, U = PIECES;
    const Side& s = a.side[blockIdx.y];
    const uint8_t* const codes = s.codes + blockIdx.z * a.code_bs;
    const float* const scales = s.scale + blockIdx.z * a.scale_bs;
    T* const out = static_cast<T*>(s.rows) + blockIdx.z * a.rows_bs;
    const size_t i0 = (size_t)blockIdx.x * (THREADS * U) + threadIdx.x, all = (size_t)a.rows * a.Hkv * CPR;
    Codes<VEC> c[U];
    float scale[U];
    size_t to[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const size_t i = i0 + u * THREADS;             // piece of the destination: (row, head, column)
        to[u] = ~(size_t)0;
        if (i >= all) continue;
        const int rh = (int)(i / CPR), col = (int)(i % CPR);
        const int r = fast_div(rh, a.dHkv), h = rh - r * a.Hkv;
        const size_t row = (size_t)a.row0 + r;
        c[u] = load_codes<VEC>(codes + ((size_t)h * a.capacity + row) * D + col * VEC);
        scale[u] = scales[(size_t)h * (a.capacity / QB) + row / QB];
        to[u] = (size_t)r * s.row_stride + h * D + col * VEC;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (to[u] == ~(size_t)0) continue;
        float x[VEC];
        decode<VEC>(c[u], scale[u], x);
        *reinterpret_cast<u32x4*>(out + to[u]) = narrow(x);
    }
}

long long row_stride(const fdd_quant_cache& c, long long stride) { return stride ? stride : (long long)c.Hkv * c.D; }

template <typename Args>
void set_sides(Args* a, const fdd_quant_cache& c, int row0, const fdd_quant_rows& r)
{
    a->side[0] = {r.k, row_stride(c, r.k_row_stride), static_cast<uint8_t*>(c.k), c.k_scale};
    a->side[1] = {r.v, row_stride(c, r.v_row_stride), static_cast<uint8_t*>(c.v), c.v_scale};
    a->Hkv = c.Hkv;
    a->capacity = c.capacity;
    a->row0 = row0;
    a->rows = r.rows;
}

}  // namespace

hipError_t launch_quantize(const fdd_quant_cache& c, int row0, const fdd_quant_rows& src, hipStream_t s)
{
    QuantArgs a;
    set_sides(&a, c, row0, src);
    const dim3 grid((unsigned)((row0 + (long long)src.rows + QB - 1) / QB - row0 / QB), (unsigned)c.Hkv, 2);
    if (src.dtype == FDD_BF16) {
        if (c.D == 128) hipLaunchKernelGGL((quantize_kernel<128, uint16_t>), grid, dim3(THREADS), 0, s, a);
        else hipLaunchKernelGGL((quantize_kernel<64, uint16_t>), grid, dim3(THREADS), 0, s, a);
    } else {
        if (c.D == 128) hipLaunchKernelGGL((quantize_kernel<128, float>), grid, dim3(THREADS), 0, s, a);
        else hipLaunchKernelGGL((quantize_kernel<64, float>), grid, dim3(THREADS), 0, s, a);
    }
    return hipGetLastError();
}

hipError_t launch_dequantize(const fdd_quant_cache& c, int row0, const fdd_quant_rows& dst, int batch, long long batch_stride, hipStream_t s)
{
    DequantArgs a;
    set_sides(&a, c, row0, dst);
    a.dHkv = make_fastdiv((uint32_t)c.Hkv);
    a.code_bs = c.batch_stride;
    a.scale_bs = c.scale_batch_stride;
    a.rows_bs = batch_stride;
    const long long pieces = (long long)dst.rows * c.Hkv * (c.D / (dst.dtype == FDD_BF16 ? 8 : 4)), per = THREADS * PIECES;
    const dim3 grid((unsigned)((pieces + per - 1) / per), 2, (unsigned)batch);
    auto go = [&](auto d, auto t) {
        constexpr int D = decltype(d)::value;
        typedef decltype(t) T;
        hipLaunchKernelGGL((dequantize_kernel<D, T>), grid, dim3(THREADS), 0, s, a);
    };
    const std::integral_constant<int, 64> d64;
    const std::integral_constant<int, 128> d128;
    if (dst.dtype == FDD_BF16) {
        if (c.D == 128) go(d128, uint16_t());
        else go(d64, uint16_t());
    } else {
        if (c.D == 128) go(d128, float());
        else go(d64, float());
    }
    return hipGetLastError();
}

}  // namespace fdd

using namespace fdd;

#define fail set_error

namespace {

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

fdd_status check_cache(const fdd_quant_cache* c, const char* fn)
{
    if (!c) return fail(FDD_ERR_NULL, "%s: cache is NULL", fn);
    if (c->Hkv <= 0 || c->D <= 0 || c->capacity <= 0 || c->capacity % QB)
        return fail(FDD_ERR_SHAPE, "%s: Hkv and D of the cache must be positive and its capacity a positive multiple of %d (got Hkv=%d D=%d capacity=%d)",
                    fn, QB, c->Hkv, c->D, c->capacity);
    if (c->D != 64 && c->D != 128) return fail(FDD_ERR_UNSUPPORTED, "%s: head size D=%d not supported (64 or 128)", fn, c->D);
    if (c->Hkv > 65535 || (long long)c->Hkv * c->capacity >= (1ll << 31)) return fail(FDD_ERR_SHAPE, "%s: the cache's Hkv*capacity is too large", fn);
    if (c->reserved != 0) return fail(FDD_ERR_UNSUPPORTED, "%s: reserved field of the cache must be 0", fn);
    if (!c->k || !c->v || !c->k_scale || !c->v_scale) return fail(FDD_ERR_NULL, "%s: k, v, k_scale and v_scale of the cache must not be NULL", fn);
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4))
        return fail(FDD_ERR_UNSUPPORTED, "%s: codes must be 16-byte aligned and scales 4-byte aligned", fn);
    return FDD_OK;
}

bool overlap(const void* p, unsigned long long n, const void* q, unsigned long long m)
{
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return a < b + m && b < a + n;
}

fdd_status check_rows(const fdd_quant_cache* c, int row0, const fdd_quant_rows* r, const char* fn)
{
    fdd_status st = check_cache(c, fn);
    if (st != FDD_OK) return st;
    if (!r) return fail(FDD_ERR_NULL, "%s: rows are NULL", fn);
    if (row0 < 0 || r->rows < 0 || (long long)row0 + r->rows > c->capacity)
        return fail(FDD_ERR_SHAPE, "%s: need row0 >= 0, rows >= 0 and row0 + rows <= capacity (got row0=%d rows=%d capacity=%d)", fn, row0, r->rows, c->capacity);
    if (r->dtype != FDD_F32 && r->dtype != FDD_BF16) return fail(FDD_ERR_DTYPE, "%s: dtype %d is neither FDD_F32 nor FDD_BF16", fn, r->dtype);
    if (r->rows == 0) return FDD_OK;
    if (!r->k || !r->v) return fail(FDD_ERR_NULL, "%s: k and v must not be NULL", fn);
    if (!aligned(r->k, 16) || !aligned(r->v, 16)) return fail(FDD_ERR_UNSUPPORTED, "%s: k and v must be 16-byte aligned", fn);
    const long long es = r->dtype == FDD_BF16 ? 2 : 4, row = (long long)c->Hkv * c->D;
    unsigned long long span[2];
    const long long strides[2] = {row_stride(*c, r->k_row_stride), row_stride(*c, r->v_row_stride)};
    for (int i = 0; i < 2; ++i) {
        if (strides[i] < row || strides[i] > (1ll << 28) || strides[i] * es % 16)
            return fail(FDD_ERR_SHAPE, "%s: a row stride of %lld must be at least %lld elements, at most 2^28, and a multiple of 16 bytes", fn, strides[i], row);
        span[i] = (unsigned long long)(((r->rows - 1) * strides[i] + row) * es);
    }
    const unsigned long long codes = (unsigned long long)row * c->capacity, scales = (unsigned long long)c->Hkv * (c->capacity / QB) * 4;
    const void* mine[2] = {r->k, r->v};
    for (int i = 0; i < 2; ++i)
        if (overlap(mine[i], span[i], c->k, codes) || overlap(mine[i], span[i], c->v, codes) || overlap(mine[i], span[i], c->k_scale, scales) ||
            overlap(mine[i], span[i], c->v_scale, scales))
            return fail(FDD_ERR_UNSUPPORTED, "%s: the rows overlap the cache", fn);
    return FDD_OK;
}

// Whether a row of k and a row of v share bytes: they must not where both are written.  (Rows may interleave, as parts of wider ones.)
bool rows_meet(const fdd_quant_cache& c, const fdd_quant_rows& r)
{
    const long long es = r.dtype == FDD_BF16 ? 2 : 4, row = (long long)c.Hkv * c.D * es, n = r.rows;
    const long long sk = row_stride(c, r.k_row_stride) * es, sv = row_stride(c, r.v_row_stride) * es;
    if (!overlap(r.k, (unsigned long long)((n - 1) * sk + row), r.v, (unsigned long long)((n - 1) * sv + row))) return false;
    const long long apart = (long long)(reinterpret_cast<uintptr_t>(r.v) - reinterpret_cast<uintptr_t>(r.k));
    // rows i of k whose neighbours in v have to be looked at: with equal strides only i - j counts
    const bool equal = sk == sv;
    for (long long i = 0; i < (equal ? 1 : n); ++i) {
        const long long to = i * sk - apart, j0 = to >= 0 ? to / sv : -((-to + sv - 1) / sv);      // the last row of v that starts at row i of k or in front of it
        for (long long j = j0; j <= j0 + 1; ++j)
            if (j >= (equal ? 1 - n : 0) && j < n && std::llabs(j * sv - to) < row) return true;
    }
    return false;
}

size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

// Bytes of one of K and V of a call's prefix in the call's type, over all problems of its batch
size_t plain_bytes(const fdd_attn_params& p)
{
    return round256((size_t)(p.batch > 1 ? p.batch : 1) * p.L * p.Hkv * p.D * (p.dtype == FDD_BF16 ? 2 : 4));
}

// The same call with the prefix as rows of its own type, which lie at the start of the workspace
fdd_attn_params plain_call(const fdd_attn_params& p)
{
    fdd_attn_params q = p;
    const size_t kv = plain_bytes(p);
    char* const ws = static_cast<char*>(p.workspace);
    q.prefix_batch_stride = (int64_t)p.L * p.Hkv * p.D;
    if (p.L > 0 && ws) {
        q.prefix_k = ws;
        q.prefix_v = ws + kv;
    }
    q.workspace = ws && p.workspace_bytes > 2 * kv ? ws + 2 * kv : nullptr;
    q.workspace_bytes = q.workspace ? p.workspace_bytes - 2 * kv : 0;
    return q;
}

// Whether a call converts the prefix tile by tile, in the attention kernel, and its plan.
bool plan_by_tile(const fdd_attn_params& p, AttnPlan* plan)
{
    if (p.dtype != FDD_BF16) return false;
    make_attn_plan(p, plan);
    plan->packed = false;
    plan->ws_vt_bytes = 0;
    plan->ws_ml_bytes *= 2;       // (with a factor of the row's averages beside m and l)
    return true;
}

const char* const kAttn = "fdd_block_attn_quant";

}  // namespace

extern "C" {

fdd_status fdd_prefix_quantize(const fdd_quant_cache* cache, int32_t row0, const fdd_quant_rows* src, void* stream)
{
    fdd_status st = check_rows(cache, row0, src, "fdd_prefix_quantize");
    if (st != FDD_OK || src->rows == 0) return st;
    const unsigned long long codes = (unsigned long long)cache->Hkv * cache->capacity * cache->D, scales = (unsigned long long)cache->Hkv * (cache->capacity / QB) * 4;
    const struct { const void* p; unsigned long long bytes; } arrays[] = {{cache->k, codes}, {cache->v, codes}, {cache->k_scale, scales}, {cache->v_scale, scales}};
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < i; ++j)
            if (overlap(arrays[i].p, arrays[i].bytes, arrays[j].p, arrays[j].bytes))
                return fail(FDD_ERR_UNSUPPORTED, "fdd_prefix_quantize: arrays of the cache overlap");
    hipError_t e = launch_quantize(*cache, row0, *src, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return fail(FDD_ERR_LAUNCH, "fdd_prefix_quantize: launch failed: %s", hipGetErrorString(e));
    return FDD_OK;
}

fdd_status fdd_prefix_dequantize(const fdd_quant_cache* cache, int32_t row0, const fdd_quant_rows* dst, void* stream)
{
    fdd_status st = check_rows(cache, row0, dst, "fdd_prefix_dequantize");
    if (st != FDD_OK || dst->rows == 0) return st;
    if (rows_meet(*cache, *dst)) return fail(FDD_ERR_UNSUPPORTED, "fdd_prefix_dequantize: rows of k and v overlap");
    hipError_t e = launch_dequantize(*cache, row0, *dst, 1, 0, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return fail(FDD_ERR_LAUNCH, "fdd_prefix_dequantize: launch failed: %s", hipGetErrorString(e));
    return FDD_OK;
}

size_t fdd_block_attn_quant_workspace(const fdd_attn_params* p)
{
    if (check_attn_shape(p, kAttn, false) != FDD_OK) return 0;
    AttnPlan plan;
    if (plan_by_tile(*p, &plan)) return plan.ws_o_bytes + plan.ws_ml_bytes;
    const fdd_attn_params q = plain_call(*p);
    return 2 * plain_bytes(*p) + fdd_block_attn_workspace(&q);
}

fdd_status fdd_block_attn_quant(const fdd_attn_params* p, const fdd_quant_cache* cache)
{
    fdd_status st = check_attn_shape(p, kAttn, false);
    if (st != FDD_OK) return st;
    if (p->prefix_k || p->prefix_v || p->prefix_v_packed)
        return fail(FDD_ERR_UNSUPPORTED, "%s: prefix_k, prefix_v and prefix_v_packed must be NULL (the prefix is in the cache)", kAttn);
    st = check_attn_pointers(p, kAttn, false);
    if (st != FDD_OK) return st;
    if (p->L > 0) {
        st = check_cache(cache, kAttn);
        if (st != FDD_OK) return st;
        if (cache->Hkv != p->Hkv || cache->D != p->D || p->L > cache->capacity)
            return fail(FDD_ERR_SHAPE, "%s: a cache of Hkv=%d D=%d capacity=%d does not fit Hkv=%d D=%d L=%d", kAttn, cache->Hkv, cache->D, cache->capacity,
                        p->Hkv, p->D, p->L);
        if (p->batch > 1 && (cache->batch_stride < (long long)p->Hkv * cache->capacity * p->D || cache->batch_stride % 16 ||
                             cache->scale_batch_stride < (long long)p->Hkv * (cache->capacity / QB)))
            return fail(FDD_ERR_SHAPE, "%s: batch_stride and scale_batch_stride of the cache must hold one problem's, codes 16-byte aligned", kAttn);
    }
    const size_t need = fdd_block_attn_quant_workspace(p);
    if (need > 0) {
        if (!p->workspace) return fail(FDD_ERR_WORKSPACE, "%s: workspace is NULL, %zu bytes needed", kAttn, need);
        if (!aligned(p->workspace, 256)) return fail(FDD_ERR_WORKSPACE, "%s: workspace must be 256-byte aligned", kAttn);
        if (p->workspace_bytes < need) return fail(FDD_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", kAttn, p->workspace_bytes, need);
    }
    const hipStream_t stream = static_cast<hipStream_t>(p->stream);
    AttnPlan plan;
    if (plan_by_tile(*p, &plan)) {
        const float scale = p->scale > 0.f ? p->scale : 1.f / std::sqrt((float)p->D);
        hipEvent_t start, stop;
        attn_events(&start, &stop);
        hipError_t e = launch_attn_quant(*p, cache, plan, scale, stream, start);
        if (e == hipSuccess && stop) e = hipEventRecord(stop, stream);
        if (e == hipSuccess && plan.ws_o_bytes > 0) e = launch_attn_merge_quant(*p, plan, scale, stream);
        if (e != hipSuccess) return fail(FDD_ERR_LAUNCH, "%s: launch failed: %s", kAttn, hipGetErrorString(e));
        return FDD_OK;
    }
    const fdd_attn_params q = plain_call(*p);
    if (p->L > 0) {
        fdd_quant_rows rows = {const_cast<void*>(q.prefix_k), const_cast<void*>(q.prefix_v), 0, 0, p->L, p->dtype};
        hipError_t e = launch_dequantize(*cache, 0, rows, p->batch > 1 ? p->batch : 1, q.prefix_batch_stride, stream);
        if (e != hipSuccess) return fail(FDD_ERR_LAUNCH, "%s: launch failed: %s", kAttn, hipGetErrorString(e));
    }
    return fdd_block_attn(&q);
}

}  // extern "C"
