// Rotary positions (fdd_rope), rows that join a paged cache with the rotation on the way (fdd_paged_append), and what tokens of a
// tree see (fdd_tree_mask).
//
// A pair (x, y) of channels becomes magnitude (x cos a - y sin a, y cos a + x sin a), a = p w.  In fp32 p w is off by 2^-25 of itself,
// 0.06 radians at p = 10^6; the frequency is therefore a fraction of a turn with 64 bits, whose product with an integer position
// drops the whole turns by itself.  The quarter turns come off as bits too, and sine and cosine are their Taylor polynomials in
// |x| <= pi / 4 (degrees 9 and 10, below 2^-25 from the functions), so that one call serves both.
//
// Rows are moved once: large calls are bound by bytes, small ones by a launch.  A thread has 16 bytes of each half of a head's pairs and takes up
// to four heads of a row, which share the angles (their 20 instructions a pair would otherwise weigh as much as the bytes).  16384
// rows of 28 + 4 heads of 128 in bf16: 47.7 us, 5.6 TB/s (a copy of 1 GiB reaches 5.2); 32 rows 3.2 us from a graph.  Append, 4 prompts
// of up to 8192 rows of 4 x 128: 19.3 us, 5.2 TB/s; 16 paths of up to 32 rows 3.1 us from a graph.  fp32: 8192 rows of 28 + 4 heads 46.8 us, 4 prompts of up to 4096 rows
// 19.2.  Where the halves of the rotated channels, or the rows, are not whole pieces of 16 bytes, a thread moves an element at a time: 16384 rows in bf16
// with 24 of 128 channels rotated 134 us, 2.0 TB/s.
#include <type_traits>

#include "paged.h"

namespace fdd {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int THREADS = 256;

// sine and cosine of 2 pi `turn` / 2^64, times m
__device__ __forceinline__ void sin_cos(uint64_t turn, float m, float* s, float* c)
{
    const uint64_t quarter = turn + (1ull << 61);                    // to the nearest quarter turn
    const int q = (int)(quarter >> 62);
    const int32_t rest = (int32_t)((turn - ((uint64_t)q << 62)) >> 32);      // of a turn, * 2^32: -2^29 .. 2^29
    // radians: the upper 24 and the lower 6 bits of `rest` are exact in fp32, 2 pi * 2^-32 is hi + lo
    constexpr double unit = 6.283185307179586476925 / 4294967296.0;
    constexpr float hi = (float)unit, lo = (float)(unit - (double)hi);
    const float a = (float)(rest & ~63), b = (float)(rest & 63);
    const float x = fmaf(a, hi, fmaf(a, lo, b * hi));
    const float z = x * x;
    float ps = fmaf(z, 1.f / 362880.f, -1.f / 5040.f);
    ps = fmaf(ps, z, 1.f / 120.f);
    ps = fmaf(ps, z, -1.f / 6.f);
    const float sine = fmaf(ps * z, x, x);
    float pc = fmaf(z, -1.f / 3628800.f, 1.f / 40320.f);
    pc = fmaf(pc, z, -1.f / 720.f);
    pc = fmaf(pc, z, 1.f / 24.f);
    pc = fmaf(pc, z, -0.5f);
    const float cosine = fmaf(pc, z, 1.f);
    // q quarter turns on: (c, s) -> (-s, c)
    const float u = q & 1 ? sine : cosine, v = q & 1 ? cosine : sine;
    *c = (q + 1) & 2 ? -u * m : u * m;
    *s = q & 2 ? -v * m : v * m;
}

// `n` elements of type T at any alignment of theirs, as fp32
template <typename T, int N>
struct Piece {
    T x[N];
};
__device__ __forceinline__ float to_f32(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }
__device__ __forceinline__ float to_f32(float x) { return x; }
template <typename T>
__device__ __forceinline__ T from_f32(float x)
{
    if constexpr (std::is_same<T, float>::value) return x;
    else return __builtin_bit_cast(uint16_t, (__bf16)x);
}
// How large calls move their bytes: past the L2s (32 MB in all), which what they write does not fit, nor anything that a call behind
// could use.  us, from a graph, arrays in rotation, bf16: 16384 rows of 32 heads of 128 rotated (268 MB) 53.1 as they come, 49.5 with such
// stores, 47.3 with such loads too; 4 prompts of up to 8192 rows of 4 x 128 into pages (101 MB) 25.5, 20.0 and 24.4.
enum Way { CACHED, STREAM_STORES, STREAM };
inline Way way_of(long long bytes_written, Way large) { return bytes_written > (32ll << 20) ? large : CACHED; }

// 16 bytes and more at once where rows are 16-byte aligned
template <typename T, int N, bool VEC, int WAY>
__device__ __forceinline__ Piece<T, N> load(const T* p)
{
    Piece<T, N> r;
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < N * (int)sizeof(T) / 16; ++i) {
            const u32x4* const at = reinterpret_cast<const u32x4*>(p) + i;
            const u32x4 w = WAY == STREAM ? __builtin_nontemporal_load(at) : *at;
            __builtin_memcpy(reinterpret_cast<char*>(&r) + i * 16, &w, 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) r.x[i] = p[i];
    }
    return r;
}
template <typename T, int N, bool VEC, int WAY>
__device__ __forceinline__ void store(T* p, const Piece<T, N>& r)
{
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < N * (int)sizeof(T) / 16; ++i) {
            u32x4 w;
            __builtin_memcpy(&w, reinterpret_cast<const char*>(&r) + i * 16, 16);
            u32x4* const at = reinterpret_cast<u32x4*>(p) + i;
            if constexpr (WAY != CACHED) __builtin_nontemporal_store(w, at);
            else *at = w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = r.x[i];
    }
}

// One head's share of a thread.  A thread takes VE pairs (or, behind them, VP channels that stay) of every head that it has: the
// angles are worked out once for all of them.  VEC: 16 bytes at a time; otherwise a pair, or a channel.
template <typename T, bool VEC, int WAY>
struct Unit {
    static constexpr int VE = VEC ? 16 / (int)sizeof(T) : 1;
    float c[VE], s[VE];
    int first;          // first pair, or channel where nothing turns
    bool turns;

    __device__ __forceinline__ void set(int u, int pairs, int rot_dim, const uint64_t* table, int position, float magnitude, bool inverse)
    {
        const int n_turn = pairs / VE;
        turns = u < n_turn;
        first = turns ? u * VE : rot_dim + (u - n_turn) * VE;
        if (!turns) return;
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            sin_cos((uint64_t)(int64_t)position * table[first + i], magnitude, &s[i], &c[i]);
            if (inverse) s[i] = -s[i];
        }
    }
    // what a head has at this unit, and what becomes of it
    __device__ __forceinline__ Piece<T, 2 * VE> read(const T* x, int pairs, bool interleaved) const
    {
        Piece<T, 2 * VE> both;
        if (turns && interleaved) return load<T, 2 * VE, VEC, WAY>(x + 2 * first);
        const Piece<T, VE> a = load<T, VE, VEC, WAY>(x + first);
        Piece<T, VE> b = a;
        if (turns) b = load<T, VE, VEC, WAY>(x + pairs + first);
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            both.x[i] = a.x[i];
            both.x[VE + i] = b.x[i];
        }
        return both;
    }
    __device__ __forceinline__ void write(const Piece<T, 2 * VE>& both, T* y, int pairs, bool interleaved) const
    {
        Piece<T, 2 * VE> r = both;
        if (turns)
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                const float u = to_f32(interleaved ? both.x[2 * i] : both.x[i]), v = to_f32(interleaved ? both.x[2 * i + 1] : both.x[VE + i]);
                const T p = from_f32<T>(fmaf(u, c[i], -(v * s[i]))), q = from_f32<T>(fmaf(v, c[i], u * s[i]));
                r.x[interleaved ? 2 * i : i] = p;
                r.x[interleaved ? 2 * i + 1 : VE + i] = q;
            }
        if (turns && interleaved) {
            store<T, 2 * VE, VEC, WAY>(y + 2 * first, r);
            return;
        }
        Piece<T, VE> a, b;
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            a.x[i] = r.x[i];
            b.x[i] = r.x[VE + i];
        }
        store<T, VE, VEC, WAY>(y + first, a);
        if (turns) store<T, VE, VEC, WAY>(y + pairs + first, b);
    }
};

// f(h) for the heads group, group + groups, .. below H, HEADS of them at a time: all reads of these come before the first write.
constexpr int HEADS = 4;
template <typename P, typename Read, typename Write>
__device__ __forceinline__ void each_head(int group, int groups, int H, const Read& read, const Write& write)
{
    int h = group;
    for (; h + (HEADS - 1) * groups < H; h += HEADS * groups) {
        P x[HEADS];
#pragma unroll
        for (int i = 0; i < HEADS; ++i) x[i] = read(h + i * groups);
#pragma unroll
        for (int i = 0; i < HEADS; ++i) write(h + i * groups, x[i]);
    }
    for (; h < H; h += groups) write(h, read(h));
}

// units of a head: VE pairs each, then VE channels each
template <typename T, bool VEC>
int units_of(int rot_dim, int D)
{
    constexpr int VE = Unit<T, VEC, CACHED>::VE;
    return rot_dim / 2 / VE + (D - rot_dim) / VE;
}

struct RopeArgs {
    const void* q;
    const void* k;
    void* q_out;
    void* k_out;
    long long q_stride, k_stride, q_out_stride, k_out_stride;
    const uint64_t* turns;
    const int32_t* positions;
    int total;              // threads: rows * groups * units
    int Hq, H, D;           // H: heads of q and k
    int groups, units;      // a thread has heads group, group + groups, ..
    int pairs, rot_dim, interleaved, inverse;
    float magnitude;
    FastDiv dUnits, dGroups;
};

template <typename T, bool VEC, bool INTERLEAVED, int WAY>
__global__ __launch_bounds__(THREADS) void rope_kernel(RopeArgs a)
{
    const int t = (int)(blockIdx.x * THREADS + threadIdx.x);
    if (t >= a.total) return;
    const int rest = fast_div(t, a.dUnits), u = t - rest * a.units;
    const int row = fast_div(rest, a.dGroups), group = rest - row * a.groups;
    Unit<T, VEC, WAY> unit;
    unit.set(u, a.pairs, a.rot_dim, a.turns, a.positions[row], a.magnitude, a.inverse);
    const bool interleaved = INTERLEAVED;
    each_head<Piece<T, 2 * Unit<T, VEC, WAY>::VE>>(
        group, a.groups, a.H,
        [&](int h) {
            const T* const x = h >= a.Hq ? static_cast<const T*>(a.k) + row * a.k_stride + (long long)(h - a.Hq) * a.D : static_cast<const T*>(a.q) + row * a.q_stride + (long long)h * a.D;
            return unit.read(x, a.pairs, interleaved);
        },
        [&](int h, const Piece<T, 2 * Unit<T, VEC, WAY>::VE>& x) {
            T* const y = h >= a.Hq ? static_cast<T*>(a.k_out) + row * a.k_out_stride + (long long)(h - a.Hq) * a.D : static_cast<T*>(a.q_out) + row * a.q_out_stride + (long long)h * a.D;
            unit.write(x, y, a.pairs, interleaved);
        });
}

struct AppendArgs {
    const void* k;
    const void* v;
    void* k_pages;
    void* v_pages;
    long long k_stride, v_stride;
    const int32_t* table;
    const int32_t* lens;
    const int32_t* positions;
    const int32_t* rows;
    const int32_t* n_rows;
    const uint64_t* turns;
    int total;                  // threads: N * B * groups * (units + V pieces)
    int B, pages, page_shift, max_pages, Hkv, D;
    int groups, units, all;     // units of k, and with the pieces of v
    int pairs, rot_dim, interleaved;
    float magnitude;
    FastDiv dAll, dGroups, dB;
};

template <typename T, bool VEC, bool INTERLEAVED, int WAY>
__global__ __launch_bounds__(THREADS) void append_kernel(AppendArgs a)
{
    constexpr int V16 = 16 / (int)sizeof(T);
    const int t = (int)(blockIdx.x * THREADS + threadIdx.x);
    if (t >= a.total) return;
    int rest = fast_div(t, a.dAll);
    const int u = t - rest * a.all;
    const int nb = fast_div(rest, a.dGroups), group = rest - nb * a.groups;
    const int n = fast_div(nb, a.dB), j = nb - n * a.B;
    if (a.n_rows && j >= a.n_rows[n]) return;
    const int src = a.rows ? a.rows[nb] : j;
    if (src < 0 || src >= a.B) return;
    const int capacity = a.max_pages << a.page_shift;
    const int slot = min(max(a.lens[n], 0), capacity) + j;
    if (slot >= capacity) return;
    const int page = a.table[(long long)n * a.max_pages + (slot >> a.page_shift)];
    if (page < 0 || page >= a.pages) return;
    const long long token = (long long)n * a.B + src;
    const long long head0 = (((long long)page * a.Hkv) << a.page_shift) + (slot & ((1 << a.page_shift) - 1));     // row of head 0 in the pool
    if (u < a.units) {
        const T* const x = static_cast<const T*>(a.k) + token * a.k_stride;
        T* const y = static_cast<T*>(a.k_pages) + head0 * a.D;
        Unit<T, VEC, WAY> unit;
        unit.set(u, a.pairs, a.rot_dim, a.turns, a.positions ? a.positions[token] : slot, a.magnitude, false);
        const bool interleaved = INTERLEAVED;
        each_head<Piece<T, 2 * Unit<T, VEC, WAY>::VE>>(
            group, a.groups, a.Hkv, [&](int h) { return unit.read(x + h * a.D, a.pairs, interleaved); },
            [&](int h, const Piece<T, 2 * Unit<T, VEC, WAY>::VE>& z) { unit.write(z, y + (((long long)h * a.D) << a.page_shift), a.pairs, interleaved); });
    } else {
        const int at = (u - a.units) * V16;
        const T* const x = static_cast<const T*>(a.v) + token * a.v_stride + at;
        T* const y = static_cast<T*>(a.v_pages) + head0 * a.D + at;
        each_head<Piece<T, V16>>(
            group, a.groups, a.Hkv, [&](int h) { return load<T, V16, true, WAY>(x + h * a.D); },
            [&](int h, const Piece<T, V16>& z) { store<T, V16, true, WAY>(y + (((long long)h * a.D) << a.page_shift), z); });
    }
}

// One workgroup per request.  A token's ancestors: its own, and those of the one that a pointer names; the pointers' distances
// double from round to round, so that ceil(log2 B) rounds reach every root (walking from parent to parent takes as many LDS
// latencies as the tree is deep: 10.8 us for 64 trees of 256 tokens, 170 deep; as it is 4.4, one of 16 tokens 1.8, of a call's 4.3 from the host).  Bound by the rounds'
// barriers.  WORDS: of a token's bits.
struct TreeArgs {
    const int32_t* parents;
    long long parents_stride;
    const int32_t* lens;
    const int32_t* n_tokens;
    uint64_t* mask;
    int32_t* positions;
    int B;
};

template <int WORDS, int MAX_B>
__global__ __launch_bounds__(MAX_B) void tree_mask_kernel(TreeArgs a)
{
    __shared__ uint64_t bits[MAX_B][WORDS];
    __shared__ int32_t jump[MAX_B];
    const int n = blockIdx.x, i = threadIdx.x, words = (a.B + 63) >> 6;
    const int there = a.n_tokens ? min(a.n_tokens[n], a.B) : a.B;
    const bool mine = i < there;
    int at = mine && i > 0 ? parent_of(i, a.parents[n * a.parents_stride + i]) : -1;
    const int len = a.lens ? a.lens[n] : 0;
    uint64_t b[WORDS];
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
        b[w] = mine && (i >> 6) == w ? 1ull << (i & 63) : 0ull;
        bits[i][w] = b[w];
    }
    jump[i] = at;
    __syncthreads();
    for (int far = 1; far < there; far *= 2) {
        int next = -1;
        if (at >= 0) {
#pragma unroll
            for (int w = 0; w < WORDS; ++w) b[w] |= bits[at][w];
            next = jump[at];
        }
        at = next;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WORDS; ++w) bits[i][w] = b[w];
        jump[i] = at;
        __syncthreads();
    }
    if (i >= a.B) return;
    int steps = -1;
#pragma unroll
    for (int w = 0; w < WORDS; ++w) {
        steps += __builtin_popcountll(b[w]);
        if (a.mask && w < words) a.mask[((long long)n * a.B + i) * words + w] = b[w];
    }
    if (a.positions) a.positions[(long long)n * a.B + i] = mine ? len + steps : 0;
}

}  // namespace
}  // namespace fdd

using namespace fdd;

#define fail set_error

fdd_status fdd::check_paged_cache(const fdd_paged_cache* c, const char* fn)
{
    if (!c) return fail(FDD_ERR_NULL, "%s: cache is NULL", fn);
    if (c->N <= 0 || c->pages <= 0 || c->max_pages <= 0 || c->Hkv <= 0)
        return fail(FDD_ERR_SHAPE, "%s: N, pages, max_pages and Hkv of the cache must be positive (got N=%d pages=%d max_pages=%d Hkv=%d)", fn, c->N, c->pages,
                    c->max_pages, c->Hkv);
    if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)))
        return fail(FDD_ERR_UNSUPPORTED, "%s: page_size=%d must be a power of two from 16 to 1024", fn, c->page_size);
    if (c->D != 64 && c->D != 128) return fail(FDD_ERR_UNSUPPORTED, "%s: head size D=%d not supported (64 or 128)", fn, c->D);
    if (c->dtype != FDD_F32 && c->dtype != FDD_BF16) return fail(FDD_ERR_DTYPE, "%s: dtype %d is neither FDD_F32 nor FDD_BF16", fn, c->dtype);
    if ((long long)c->max_pages * c->page_size >= (1ll << 30)) return fail(FDD_ERR_SHAPE, "%s: max_pages*page_size must be below 2^30", fn);
    if (c->Hkv > 65535 || (long long)c->N * c->Hkv >= (1ll << 28) || (long long)c->pages * c->Hkv >= (1ll << 32))
        return fail(FDD_ERR_SHAPE, "%s: N*Hkv or pages*Hkv too large", fn);
    if ((long long)c->page_size * c->Hkv * c->D * 4 >= (1ll << 31)) return fail(FDD_ERR_SHAPE, "%s: a page must stay below 2 GiB", fn);
    if (c->reserved != 0) return fail(FDD_ERR_UNSUPPORTED, "%s: reserved field of the cache must be 0", fn);
    if (!c->k || !c->v || !c->page_table || !c->lens) return fail(FDD_ERR_NULL, "%s: k, v, page_table and lens of the cache must not be NULL", fn);
    if (!aligned_to(c->k, 16) || !aligned_to(c->v, 16) || !aligned_to(c->page_table, 4) || !aligned_to(c->lens, 4))
        return fail(FDD_ERR_UNSUPPORTED, "%s: pages must be 16-byte aligned, page_table and lens 4-byte aligned", fn);
    return FDD_OK;
}

fdd_status fdd::check_token_stride(long long stride, long long token, int dtype, const char* what, const char* fn)
{
    if (stride == 0) return FDD_OK;
    if (stride < token || stride > (1ll << 28) || stride * dtype_bytes(dtype) % 16)
        return fail(FDD_ERR_SHAPE, "%s: %s=%lld must be at least %lld elements, at most 2^28, and a multiple of 16 bytes", fn, what, stride, token);
    return FDD_OK;
}

namespace {

fdd_status check_table(const fdd_rope_table& t, int D, const char* fn)
{
    if (!t.turns) return fail(FDD_ERR_NULL, "%s: turns of the table is NULL", fn);
    if (t.rot_dim < 2 || t.rot_dim % 2 || t.rot_dim > D) return fail(FDD_ERR_SHAPE, "%s: rot_dim=%d must be even, from 2 to D=%d", fn, t.rot_dim, D);
    if (t.interleaved != 0 && t.interleaved != 1) return fail(FDD_ERR_UNSUPPORTED, "%s: interleaved=%d is neither 0 nor 1", fn, t.interleaved);
    if (!std::isfinite(t.magnitude)) return fail(FDD_ERR_UNSUPPORTED, "%s: magnitude is not finite", fn);
    if (t.reserved != 0) return fail(FDD_ERR_UNSUPPORTED, "%s: reserved field of the table must be 0", fn);
    if (!aligned_to(t.turns, 8)) return fail(FDD_ERR_UNSUPPORTED, "%s: turns must be 8-byte aligned", fn);
    return FDD_OK;
}

// Whether a head's pairs and the channels behind them come in whole pieces of 16 bytes
bool whole_pieces(int rot_dim, int D, int dtype)
{
    const int ve = 16 / (int)dtype_bytes(dtype);
    return rot_dim / 2 % ve == 0 && (D - rot_dim) % ve == 0;
}

// Heads that a thread takes one after the other: each of them its own thread while that leaves compute units idle, four
// otherwise, which then share the angles.
int head_groups(long long rows, int heads, int units) { return rows * heads * units <= 8ll * kNumCU * THREADS ? heads : (heads + 3) / 4; }

}  // namespace

extern "C" {

fdd_status fdd_rope_turns(const fdd_rope_scaling* p, uint64_t* turns, float* magnitude)
{
    const char* const fn = "fdd_rope_turns";
    if (!p || !turns || !magnitude) return fail(FDD_ERR_NULL, "%s: params, turns and magnitude must not be NULL", fn);
    if (p->rot_dim < 2 || p->rot_dim > 1024 || p->rot_dim % 2) return fail(FDD_ERR_SHAPE, "%s: rot_dim=%d must be even, from 2 to 1024", fn, p->rot_dim);
    if (p->scaling < FDD_ROPE_NONE || p->scaling > FDD_ROPE_PARTS) return fail(FDD_ERR_UNSUPPORTED, "%s: unknown scaling %d", fn, p->scaling);
    if (!(p->base > 1.0) || !std::isfinite(p->base)) return fail(FDD_ERR_UNSUPPORTED, "%s: base must be above 1 and finite", fn);
    const bool scaled = p->scaling != FDD_ROPE_NONE, parts = p->scaling == FDD_ROPE_PARTS;
    if (scaled && (!(p->stretch >= 1.0) || !std::isfinite(p->stretch))) return fail(FDD_ERR_UNSUPPORTED, "%s: stretch must be at least 1 and finite", fn);
    if (parts && (!(p->original > 0.0) || !std::isfinite(p->original))) return fail(FDD_ERR_UNSUPPORTED, "%s: original must be positive and finite", fn);
    if (p->scaling == FDD_ROPE_BASE && p->rot_dim < 4) return fail(FDD_ERR_SHAPE, "%s: a stretched base needs a rot_dim of 4 or more", fn);
    const long double two_pi = 6.283185307179586476925286766559L;
    const int R = p->rot_dim;
    const long double s = scaled ? (long double)p->stretch : 1.0L;
    const long double base = p->scaling == FDD_ROPE_BASE ? (long double)p->base * std::pow(s, (long double)R / (R - 2)) : (long double)p->base;
    if (!std::isfinite((double)base)) return fail(FDD_ERR_UNSUPPORTED, "%s: the stretched base is not finite", fn);
    for (int i = 0; i < R / 2; ++i) {
        long double w = std::pow(base, -2.0L * i / R);
        if (p->scaling == FDD_ROPE_LINEAR) w /= s;
        if (parts) {
            const long double rounds = (long double)p->original * w / two_pi;
            const long double g = std::fmin(1.0L, std::fmax(0.0L, (rounds - 1.0L) / 31.0L));
            w = g * w + (1.0L - g) * w / s;
        }
        turns[i] = (uint64_t)std::floor(w / two_pi * 18446744073709551616.0L + 0.5L);      // (w <= 1: below a sixth of 2^64)
    }
    *magnitude = parts ? (float)(0.1L * std::log(s) + 1.0L) : 1.f;
    return FDD_OK;
}

fdd_status fdd_rope(const fdd_rope_params* p)
{
    const char* const fn = "fdd_rope";
    if (!p) return fail(FDD_ERR_NULL, "%s: params is NULL", fn);
    if (p->rows < 0 || p->Hq <= 0 || p->D <= 0 || p->D > 1024 || (p->k && p->Hk <= 0))
        return fail(FDD_ERR_SHAPE, "%s: Hq, D and Hk must be positive, D at most 1024 and rows >= 0 (got rows=%d Hq=%d Hk=%d D=%d)", fn, p->rows, p->Hq, p->Hk, p->D);
    if (p->dtype != FDD_F32 && p->dtype != FDD_BF16) return fail(FDD_ERR_DTYPE, "%s: dtype %d is neither FDD_F32 nor FDD_BF16", fn, p->dtype);
    if (p->flags & ~FDD_ROPE_INVERSE) return fail(FDD_ERR_UNSUPPORTED, "%s: unknown bits in flags (0x%x)", fn, p->flags);
    fdd_status st = check_table(p->table, p->D, fn);
    if (st != FDD_OK) return st;
    const long long heads = (long long)p->Hq + (p->k ? p->Hk : 0);
    if (heads > 65535) return fail(FDD_ERR_SHAPE, "%s: too many heads", fn);
    if (p->rows == 0) return FDD_OK;
    if (!p->q || !p->q_out || !p->positions || (!p->k != !p->k_out)) return fail(FDD_ERR_NULL, "%s: q, q_out and positions must not be NULL, k and k_out both or neither", fn);
    const long long es = dtype_bytes(p->dtype);
    struct Array { const void* p; long long stride, row; bool out; };
    Array arrays[] = {{p->q, p->q_stride, (long long)p->Hq * p->D, false}, {p->q_out, p->q_out_stride, (long long)p->Hq * p->D, true},
                      {p->k, p->k_stride, (long long)p->Hk * p->D, false}, {p->k_out, p->k_out_stride, (long long)p->Hk * p->D, true}};
    const int n_arrays = p->k ? 4 : 2;
    bool vec = whole_pieces(p->table.rot_dim, p->D, p->dtype) && p->D * es % 16 == 0;
    for (int i = 0; i < n_arrays; ++i) {
        Array& x = arrays[i];
        if (x.stride == 0) x.stride = x.row;
        if (x.stride < x.row || x.stride > (1ll << 28)) return fail(FDD_ERR_SHAPE, "%s: a stride of %lld must be at least %lld elements and at most 2^28", fn, x.stride, x.row);
        if (!aligned_to(x.p, es)) return fail(FDD_ERR_UNSUPPORTED, "%s: arrays must be aligned to their element type", fn);
        vec = vec && aligned_to(x.p, 16) && x.stride * es % 16 == 0;
    }
    if (!aligned_to(p->positions, 4)) return fail(FDD_ERR_UNSUPPORTED, "%s: positions must be 4-byte aligned", fn);
    auto span = [&](const Array& x) { return (unsigned long long)(((long long)(p->rows - 1) * x.stride + x.row) * es); };
    for (int i = 0; i < n_arrays; ++i) {
        if (!arrays[i].out) continue;
        if (spans_overlap(arrays[i].p, span(arrays[i]), p->positions, (unsigned long long)p->rows * 4) ||
            spans_overlap(arrays[i].p, span(arrays[i]), p->table.turns, (unsigned long long)p->table.rot_dim * 4))
            return fail(FDD_ERR_UNSUPPORTED, "%s: an output overlaps positions or turns", fn);
        for (int j = 0; j < n_arrays; ++j) {
            if (i == j || !spans_overlap(arrays[i].p, span(arrays[i]), arrays[j].p, span(arrays[j]))) continue;
            if (j == i - 1 && arrays[i].p == arrays[j].p && arrays[i].stride == arrays[j].stride) continue;      // in place
            // arrays that interleave, as parts of wider rows: the same stride, and no row of one meets a row of the other
            const long long apart = (long long)(reinterpret_cast<intptr_t>(arrays[j].p) - reinterpret_cast<intptr_t>(arrays[i].p)), wide = arrays[i].stride * es;
            const long long m = ((apart % wide) + wide) % wide;
            if (arrays[i].stride == arrays[j].stride && m >= arrays[i].row * es && m + arrays[j].row * es <= wide) continue;
            return fail(FDD_ERR_UNSUPPORTED, "%s: an output overlaps another array", fn);
        }
    }
    RopeArgs a = {};
    a.q = p->q; a.k = p->k; a.q_out = p->q_out; a.k_out = p->k_out;
    a.q_stride = arrays[0].stride; a.q_out_stride = arrays[1].stride; a.k_stride = arrays[2].stride; a.k_out_stride = arrays[3].stride;
    a.turns = p->table.turns; a.positions = p->positions;
    a.Hq = p->Hq; a.H = (int)heads; a.D = p->D;
    a.pairs = p->table.rot_dim / 2; a.rot_dim = p->table.rot_dim; a.interleaved = p->table.interleaved;
    a.inverse = p->flags & FDD_ROPE_INVERSE; a.magnitude = p->table.magnitude;
    const bool bf16 = p->dtype == FDD_BF16;
    a.units = bf16 ? (vec ? units_of<uint16_t, true>(a.rot_dim, a.D) : units_of<uint16_t, false>(a.rot_dim, a.D))
                   : (vec ? units_of<float, true>(a.rot_dim, a.D) : units_of<float, false>(a.rot_dim, a.D));
    a.groups = head_groups(p->rows, a.H, a.units);
    const long long total = (long long)p->rows * a.groups * a.units;
    if (total >= (1ll << 31) - THREADS) return fail(FDD_ERR_SHAPE, "%s: rows*heads*D too large", fn);
    a.total = (int)total;
    a.dUnits = make_fastdiv((uint32_t)a.units); a.dGroups = make_fastdiv((uint32_t)a.groups);
    const dim3 grid((unsigned)((total + THREADS - 1) / THREADS));
    const hipStream_t s = static_cast<hipStream_t>(p->stream);
    const Way way = way_of((long long)p->rows * heads * p->D * es, STREAM);
    auto run = [&](auto type, auto vector) {
        using T = decltype(type);
        constexpr bool VEC = decltype(vector)::value;
        constexpr int LARGE = VEC ? STREAM : CACHED;
        if (way == CACHED && a.interleaved) rope_kernel<T, VEC, true, CACHED><<<grid, THREADS, 0, s>>>(a);
        else if (way == CACHED) rope_kernel<T, VEC, false, CACHED><<<grid, THREADS, 0, s>>>(a);
        else if (a.interleaved) rope_kernel<T, VEC, true, LARGE><<<grid, THREADS, 0, s>>>(a);
        else rope_kernel<T, VEC, false, LARGE><<<grid, THREADS, 0, s>>>(a);
    };
    if (bf16 && vec) run(uint16_t(), std::true_type());
    else if (bf16) run(uint16_t(), std::false_type());
    else if (vec) run(float(), std::true_type());
    else run(float(), std::false_type());
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(FDD_ERR_LAUNCH, "%s: launch failed: %s", fn, hipGetErrorString(e));
    return FDD_OK;
}

fdd_status fdd_paged_append(const fdd_paged_cache* c, const fdd_paged_append_params* p)
{
    const char* const fn = "fdd_paged_append";
    fdd_status st = check_paged_cache(c, fn);
    if (st != FDD_OK) return st;
    if (!p) return fail(FDD_ERR_NULL, "%s: params is NULL", fn);
    if (p->B <= 0) return fail(FDD_ERR_SHAPE, "%s: B=%d must be positive", fn, p->B);
    if (p->reserved != 0) return fail(FDD_ERR_UNSUPPORTED, "%s: reserved field must be 0", fn);
    if (!p->k || !p->v) return fail(FDD_ERR_NULL, "%s: k and v must not be NULL", fn);
    if (!aligned_to(p->k, 16) || !aligned_to(p->v, 16) || !aligned_to(p->positions, 4) || !aligned_to(p->rows, 4) || !aligned_to(p->n_rows, 4))
        return fail(FDD_ERR_UNSUPPORTED, "%s: k and v must be 16-byte aligned, lists 4-byte aligned", fn);
    const long long es = dtype_bytes(c->dtype), token = (long long)c->Hkv * c->D, tokens = (long long)c->N * p->B;
    if ((st = check_token_stride(p->k_stride, token, c->dtype, "k_stride", fn)) != FDD_OK) return st;
    if ((st = check_token_stride(p->v_stride, token, c->dtype, "v_stride", fn)) != FDD_OK) return st;
    if (p->rope && (st = check_table(*p->rope, c->D, fn)) != FDD_OK) return st;
    if (tokens >= (1ll << 31)) return fail(FDD_ERR_SHAPE, "%s: N*B too large", fn);
    AppendArgs a = {};
    a.k_stride = token_stride(p->k_stride, token); a.v_stride = token_stride(p->v_stride, token);
    const unsigned long long pool = pool_bytes(*c);
    if (spans_overlap(c->k, pool, c->v, pool)) return fail(FDD_ERR_UNSUPPORTED, "%s: K's and V's pages overlap", fn);
    const struct { const void* p; unsigned long long bytes; } reads[] = {
        {p->k, (unsigned long long)(((tokens - 1) * a.k_stride + token) * es)}, {p->v, (unsigned long long)(((tokens - 1) * a.v_stride + token) * es)},
        {c->page_table, (unsigned long long)c->N * c->max_pages * 4}, {c->lens, (unsigned long long)c->N * 4},
        {p->positions, p->positions ? (unsigned long long)tokens * 4 : 0}, {p->rows, p->rows ? (unsigned long long)tokens * 4 : 0},
        {p->n_rows, p->n_rows ? (unsigned long long)c->N * 4 : 0}, {p->rope ? p->rope->turns : nullptr, p->rope ? (unsigned long long)p->rope->rot_dim * 4 : 0}};
    for (const auto& r : reads)
        if (spans_overlap(r.p, r.bytes, c->k, pool) || spans_overlap(r.p, r.bytes, c->v, pool)) return fail(FDD_ERR_UNSUPPORTED, "%s: an input overlaps the cache's pages", fn);
    a.k = p->k; a.v = p->v; a.k_pages = c->k; a.v_pages = c->v;
    a.table = c->page_table; a.lens = c->lens; a.positions = p->positions; a.rows = p->rows; a.n_rows = p->n_rows;
    a.B = p->B; a.pages = c->pages; a.max_pages = c->max_pages; a.Hkv = c->Hkv; a.D = c->D;
    a.page_shift = __builtin_ctz((unsigned)c->page_size);
    if (p->rope) {
        a.turns = p->rope->turns; a.rot_dim = p->rope->rot_dim; a.pairs = a.rot_dim / 2;
        a.interleaved = p->rope->interleaved; a.magnitude = p->rope->magnitude;
    }
    const bool bf16 = c->dtype == FDD_BF16, vec = whole_pieces(a.rot_dim, a.D, c->dtype);
    a.units = bf16 ? (vec ? units_of<uint16_t, true>(a.rot_dim, a.D) : units_of<uint16_t, false>(a.rot_dim, a.D))
                   : (vec ? units_of<float, true>(a.rot_dim, a.D) : units_of<float, false>(a.rot_dim, a.D));
    a.all = a.units + (int)(c->D * es / 16);
    a.groups = head_groups(tokens, c->Hkv, a.all);
    const long long total = tokens * a.groups * a.all;
    if (total >= (1ll << 31) - THREADS) return fail(FDD_ERR_SHAPE, "%s: N*B*Hkv*D too large", fn);
    a.total = (int)total;
    a.dAll = make_fastdiv((uint32_t)a.all); a.dGroups = make_fastdiv((uint32_t)a.groups); a.dB = make_fastdiv((uint32_t)a.B);
    const dim3 grid((unsigned)((total + THREADS - 1) / THREADS));
    const hipStream_t s = static_cast<hipStream_t>(p->stream);
    const Way way = way_of(2 * tokens * token * es, STREAM_STORES);
    auto run = [&](auto type, auto vector) {
        using T = decltype(type);
        constexpr bool VEC = decltype(vector)::value;
        constexpr int LARGE = VEC ? STREAM_STORES : CACHED;
        if (way == CACHED && a.interleaved) append_kernel<T, VEC, true, CACHED><<<grid, THREADS, 0, s>>>(a);
        else if (way == CACHED) append_kernel<T, VEC, false, CACHED><<<grid, THREADS, 0, s>>>(a);
        else if (a.interleaved) append_kernel<T, VEC, true, LARGE><<<grid, THREADS, 0, s>>>(a);
        else append_kernel<T, VEC, false, LARGE><<<grid, THREADS, 0, s>>>(a);
    };
    if (bf16 && vec) run(uint16_t(), std::true_type());
    else if (bf16) run(uint16_t(), std::false_type());
    else if (vec) run(float(), std::true_type());
    else run(float(), std::false_type());
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(FDD_ERR_LAUNCH, "%s: launch failed: %s", fn, hipGetErrorString(e));
    return FDD_OK;
}

fdd_status fdd_tree_mask(const fdd_tree_mask_params* p)
{
    const char* const fn = "fdd_tree_mask";
    if (!p) return fail(FDD_ERR_NULL, "%s: params is NULL", fn);
    if (p->N <= 0 || p->B <= 0) return fail(FDD_ERR_SHAPE, "%s: N and B must be positive (got N=%d B=%d)", fn, p->N, p->B);
    if (p->B > FDD_TREE_MAX) return fail(FDD_ERR_UNSUPPORTED, "%s: B=%d is above %d", fn, p->B, FDD_TREE_MAX);
    if (p->parents_stride != 0 && (p->parents_stride < p->B || p->parents_stride > (1ll << 28)))
        return fail(FDD_ERR_SHAPE, "%s: parents_stride=%lld must be 0, or at least B=%d and at most 2^28", fn, (long long)p->parents_stride, p->B);
    if (!p->parents || (!p->mask && !p->positions)) return fail(FDD_ERR_NULL, "%s: parents and one of mask and positions must not be NULL", fn);
    if (!aligned_to(p->parents, 4) || !aligned_to(p->lens, 4) || !aligned_to(p->n_tokens, 4) || !aligned_to(p->mask, 8) || !aligned_to(p->positions, 4))
        return fail(FDD_ERR_UNSUPPORTED, "%s: mask must be 8-byte aligned, the other arrays 4-byte aligned", fn);
    if (p->N >= (1 << 22) || (long long)p->N * p->B >= (1ll << 31)) return fail(FDD_ERR_SHAPE, "%s: N or N*B too large", fn);      // (a launch has at most 2^32 threads)
    const unsigned long long N = p->N, B = p->B;
    const Span outs[] = {{p->mask, N * B * ((B + 63) / 64) * 8}, {p->positions, N * B * 4}};
    const Span ins[] = {{p->parents, ((N - 1) * p->parents_stride + B) * 4}, {p->lens, N * 4}, {p->n_tokens, N * 4}};
    if (outputs_overlap(outs, ins)) return fail(FDD_ERR_UNSUPPORTED, "%s: an output overlaps another array", fn);
    TreeArgs a = {p->parents, p->parents_stride, p->lens, p->n_tokens, p->mask, p->positions, p->B};
    const dim3 grid((unsigned)p->N);
    const hipStream_t s = static_cast<hipStream_t>(p->stream);
    if (p->B <= 64) tree_mask_kernel<1, 64><<<grid, 64, 0, s>>>(a);
    else if (p->B <= 128) tree_mask_kernel<2, 128><<<grid, 128, 0, s>>>(a);
    else if (p->B <= 256) tree_mask_kernel<4, 256><<<grid, 256, 0, s>>>(a);
    else if (p->B <= 512) tree_mask_kernel<8, 512><<<grid, 512, 0, s>>>(a);
    else tree_mask_kernel<16, 1024><<<grid, 1024, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(FDD_ERR_LAUNCH, "%s: launch failed: %s", fn, hipGetErrorString(e));
    return FDD_OK;
}

}  // extern "C"
