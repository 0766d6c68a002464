// Log probability of a given token, entropy and top alternatives of rows of logits.
//
// With m the largest logit of a row, attained by entry a (any one, if there are several), y_v = (x_v - m) / temperature and
//     S = sum_{v != a} e^y_v,   U = sum_v y_v e^y_v   (the term of a is 0)
// the softmax is p_v = e^y_v / (1 + S), so
//     ln p_v = y_v - ln(1 + S),   entropy = -sum p ln p = ln(1 + S) - U / (1 + S).
// Both terms of the entropy are >= 0, and S without the largest term keeps its digits where the row is nearly certain.
//
// Bound by the bytes of the logits, which are read once, and close behind by the vector ALUs (13 instructions an entry, an exponential
// among them).  N=16, B=64, V=152064 bf16, top 5 71 to 77 us (4.4 to 4.0 TB/s); N=8, B=32 25.7, half of the rows selected 18.6, top 0 14.9; N=1, B=32 11.6; one
// piece (V=512) 4.8.  A row is cut into pieces, a workgroup each; a thread requests its part together and takes its sums as the vectors come, against a number near its largest
// entry, before it meets the others.  Entry a is left out in the end: the one thread that has it has its sums taken again, an
// entry a lane.
// A thread keeps the largest entry of each of its vectors of 16 bytes, from which the top ones are found:
//   1. T is the K-th largest of the 64 maxima of groups of 4 threads: K different entries are at least T.
//   2. The vectors that have an entry above T, little more than K in most rows, and of those whose largest is T the first K of each
//      wavefront, which have the lowest ids, are read once more, an entry a lane; entries from T on go to a list.
//   3. The place of a list entry is the number of entries ahead of it in the order (logit descending, id ascending).
//   Where the lists are too short (the largest entries of a row all lie in a few threads) they are taken out one by one.
// A row of one piece is finished by its workgroup; the pieces of other rows are joined by a second kernel, sums in fp64.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "fdd_internal.h"
#include "rows.h"
#include "wave.h"

namespace fdd {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
// 16-byte vectors a thread holds at most.  Of 4, 6, 8, 12, 16 fastest with 8 at up to 256 rows of 152064; 12 and 16 are 2 to 5 % faster
// at 1024 rows of bf16 and up to 7 % slower in others.  Pieces of two a thread or fewer have a kernel of their own, without the requests
// that bring nothing new; us with it and without: N=1, B=8, V=512 fp32 4.8 and 5.1; N=32, B=64, V=512 bf16 8.3 and 8.8; N=8, B=32, V=4001 5.6 and
// 5.9; N=1, B=32, V=50001, top 20 10.3 and 10.6 (limits of one and four instead of two: within 0.2 of it).
constexpr int MAX_NV = 8;
constexpr int FEW_NV = 2;
constexpr int MAX_TOP = FDD_LOGPROBS_MAX_TOP;
constexpr int NEAR = 128;                    // vectors of a wavefront that may hold top entries
constexpr int LIST = 1024;                   // candidates for the top entries of a piece
constexpr float LOG2E = 1.4426950408889634f;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Partial {
    float m;      // largest logit of the piece
    float s, u;   // sums of 2^y and y 2^y over the others, y = (x - m) log2(e) / temperature
    float pad;
};

struct Args {
    const void* logits;
    const int32_t* tokens;
    const uint8_t* mask;
    float* logprobs;
    float* entropy;
    int32_t* top_ids;
    float* top_logprobs;
    Partial* parts;              // [row][piece]
    uint64_t* keys;              // [row][piece][top]
    long long V;
    int rows, top, pieces, per;  // `per`: vectors of a piece
    FastDiv dPieces;
    float inv_t, c;              // 1 / temperature, log2(e) / temperature
};

// Order of (logit, id): the larger logit first, the lower id among equal ones.  As one unsigned number, larger is earlier;
// 0 stands for no entry.
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t b = __float_as_uint(x) == 0x80000000u ? 0u : __float_as_uint(x);            // (-0 counts as 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }
__device__ __forceinline__ uint64_t key_of(float x, int id) { return ((uint64_t)ordered(x) << 32) | (uint32_t)~id; }
__device__ __forceinline__ int key_id(uint64_t k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ float key_logit(uint64_t k) { return unordered((uint32_t)(k >> 32)); }

__device__ __forceinline__ float wave_max(float x)
{
    return __uint_as_float(wave_reduce(__float_as_uint(x), [](uint32_t p, uint32_t q) {
        return __float_as_uint(fmaxf(__uint_as_float(p), __uint_as_float(q)));
    }));
}
__device__ __forceinline__ float wave_sum(float x)
{
    return __uint_as_float(wave_reduce(__float_as_uint(x), [](uint32_t p, uint32_t q) {
        return __float_as_uint(__uint_as_float(p) + __uint_as_float(q));
    }));
}

template <typename T> __device__ __forceinline__ float logit(const void* x, size_t i);
template <> __device__ __forceinline__ float logit<uint16_t>(const void* x, size_t i) { return __uint_as_float((uint32_t)static_cast<const uint16_t*>(x)[i] << 16); }
template <> __device__ __forceinline__ float logit<float>(const void* x, size_t i) { return static_cast<const float*>(x)[i]; }

// the entries of a 16-byte vector
template <typename T>
__device__ __forceinline__ void widen(const u32x4& raw, float (&x)[16 / sizeof(T)])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (sizeof(T) == 2) {
            x[2 * j] = __uint_as_float(raw[j] << 16);
            x[2 * j + 1 < 16 / sizeof(T) ? 2 * j + 1 : 0] = __uint_as_float(raw[j] & 0xffff0000u);
        } else {
            x[j] = __uint_as_float(raw[j]);
        }
    }
}

constexpr uint32_t NAN_BITS = 0x7fc00000u;      // (this file is compiled for arithmetic without NaN: they are written as bits)

// What a row's outputs are made of: its largest logit and ln(1 + S); a row without a finite entry has NaN
struct RowSum {
    double lse, U, S;
    float m;
    bool empty;
};

// bits of ln p of logit x
__device__ __forceinline__ uint32_t log_prob(const RowSum& r, float x, float inv_t)
{
    const float v = (float)(((double)x - (double)r.m) * inv_t - r.lse);
    return r.empty ? NAN_BITS : __float_as_uint(v);
}

template <typename T>
__device__ __forceinline__ void write_row(const Args& a, size_t row, const RowSum& r)
{
    if (a.logprobs) {
        const int t = a.tokens[row];
        uint32_t v = 0xff800000u;                // a token outside the vocabulary: -inf
        if (t >= 0 && t < a.V) v = log_prob(r, logit<T>(a.logits, row * (size_t)a.V + t), a.inv_t);
        reinterpret_cast<uint32_t*>(a.logprobs)[row] = v;
    }
    if (a.entropy) {
        const float v = (float)(r.lse - r.U / (1.0 + r.S));
        reinterpret_cast<uint32_t*>(a.entropy)[row] = r.empty ? NAN_BITS : __float_as_uint(v);
    }
}

__device__ __forceinline__ void write_top(const Args& a, size_t row, int place, uint64_t key, const RowSum& r)
{
    a.top_ids[row * a.top + place] = key_id(key);
    reinterpret_cast<uint32_t*>(a.top_logprobs)[row * a.top + place] = log_prob(r, key_logit(key), a.inv_t);
}

__device__ __forceinline__ RowSum row_sum(float m, double s, double u)
{
    RowSum r;
    r.m = m;
    r.empty = m == -INFINITY;
    r.S = s;
    r.U = u * 0.6931471805599453;
    r.lse = log1p(r.empty ? 0.0 : r.S);
    return r;
}

constexpr float FAR = -200.f;       // 2^y is 0 from -150 on; a difference of -inf would make NaN of y 2^y

constexpr float NO_REF = -0x1.fffffep127f;      // the lowest number: no reference lies above its thread's entries, so that sums are never scaled up to another one

struct WaveSum {
    float m;          // largest entry
    float s, u;       // sums of 2^y and y 2^y, y = (x - m) c, of all threads but the first one that has m
    float os, ou;     // and of that one
    int lane;
};

// one workgroup per (row, piece); ONE: a row is one piece, and is finished here; COMPACT: workgroups are dealt to selected rows only
template <typename T, bool ONE, bool COMPACT, int NV>
__global__ __launch_bounds__(THREADS) void logprobs_kernel(Args a)
{
    constexpr int VEC = 16 / sizeof(T);
    int unit = (int)wg_id_x(), row, piece;
    if (COMPACT) {
        const int t = fast_div(unit, a.dPieces);
        piece = unit - t * a.pieces;
        row = eligible_row(a.mask, nullptr, a.rows, t);
        if (row < 0) return;
        unit = row * a.pieces + piece;
    } else {
        if (a.mask) unit = (int)unit_of_workgroup((unsigned)(a.rows * a.pieces));
        row = ONE ? unit : fast_div(unit, a.dPieces);
        piece = ONE ? 0 : unit - row * a.pieces;
        if (a.mask && a.mask[row] != 1) return;
    }
    const int tid = thread_id_x(), wave = tid >> 6, lane = tid & 63;
    __shared__ float maxima[THREADS], extras[2 * VEC];
    __shared__ WaveSum waves[WAVES];
    __shared__ RowSum sum;
    __shared__ __align__(16) float groups[WAVES][64];
    __shared__ int near[WAVES][NEAR];
    __shared__ uint64_t list[LIST];
    __shared__ int listed;
    __shared__ uint32_t bound_bits;

    // A row is its entries up to a 16-byte boundary, whole vectors, and what is left; the vectors are cut into pieces, the entries in
    // front belong to the first piece (a lane of wavefront 0 each), those behind to the last (wavefront 1).
    const size_t first = (size_t)row * (size_t)a.V;
    const int head = (int)min((long long)((0 - first) % VEC), a.V), row_vecs = (int)((a.V - head) / VEC), behind = (int)((a.V - head) % VEC);
    const int lo = piece * a.per, n_vecs = min(a.per, row_vecs - lo);
    const u32x4* const src = reinterpret_cast<const u32x4*>(static_cast<const T*>(a.logits) + first + head) + lo;
    auto id_of = [&](int i) { return head + (lo + i) * VEC; };       // id of entry 0 of vector i of the piece

    // (threads beyond the last vector read it once more and drop it: no branches between the requests, which are waited for one
    // by one then)
    u32x4 raw[NV];
    if (n_vecs > 0) {
#pragma unroll
        for (int v = 0; v < NV; ++v) raw[v] = src[min(v * THREADS + tid, n_vecs - 1)];
    }
    int extra_id = -1;
    if (wave == 0 && piece == 0 && lane < head) extra_id = lane;
    if (wave == 1 && (ONE || piece == a.pieces - 1) && lane < behind) extra_id = (int)(a.V - behind) + lane;
    const float extra_read = logit<T>(a.logits, first + max(extra_id, 0)), extra = extra_id >= 0 ? extra_read : -INFINITY;
    if (tid == 0) {
        listed = 0;
        bound_bits = ~0u;
    }
    __builtin_amdgcn_sched_barrier(0);      // all of them are requested before the first is waited for

    // ---- this thread's entries as they come: the largest of each vector, sums ------------------------------------------------------------
    // The sums are taken against a reference that is raised only when an entry is 2^64 times as probable: the sums stay far from
    // the ends of fp32's range, and the branch is rare (raised to every new largest entry it was taken by a lane of nearly
    // every wavefront at every vector).
    float vmax[NV], tmax = -INFINITY, ref = NO_REF, s = 0.f, u = 0.f;
    auto meet = [&](float largest) {
        if ((largest - ref) * a.c > 64.f) {
            const float d = fmaxf((ref - largest) * a.c, FAR), f = __builtin_amdgcn_exp2f(d);
            u = f * fmaf(d, s, u);
            s = f * s;
            ref = largest;
        }
        tmax = fmaxf(tmax, largest);
    };
    auto add = [&](float x) {
        const float y = fmaxf((x - ref) * a.c, FAR), e = __builtin_amdgcn_exp2f(y);
        s += e;
        u = fmaf(y, e, u);
    };
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        vmax[v] = -INFINITY;
        if (v * THREADS >= n_vecs) continue;
        if ((v + 1) * THREADS > n_vecs) {
            asm volatile("");           // (a branch, not a choice in every vector)
            constexpr uint32_t MISSING = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;        // -inf
            if (v * THREADS + tid >= n_vecs) raw[v] = u32x4{MISSING, MISSING, MISSING, MISSING};
        }
        float x[VEC], t;
        widen<T>(raw[v], x);
        t = x[0];
#pragma unroll
        for (int j = 1; j < VEC; ++j) t = fmaxf(t, x[j]);
        vmax[v] = t;
        meet(t);
#pragma unroll
        for (int j = 0; j < VEC; ++j) add(x[j]);
        __builtin_amdgcn_sched_barrier(0);
    }
    if (__any(extra_id >= 0)) {
        meet(extra);
        add(extra);
    }
    // this wavefront's largest entry, the first thread that has it, sums against it of the other threads
    {
        const float m = wave_max(tmax), far = m == -INFINITY ? 0.f : m;
        const int first_lane = __builtin_ctzll(__builtin_amdgcn_ballot_w64(tmax == m) | 1ull << 63);
        auto share = [&](bool in, float& ws, float& wu) {
            const float g = fmaxf((ref - far) * a.c, FAR), f = in ? __builtin_amdgcn_exp2f(g) : 0.f;
            ws = f * s;
            wu = f * fmaf(g, s, u);
        };
        float ws, wu;
        share(lane != first_lane, ws, wu);
        ws = wave_sum(ws);
        wu = wave_sum(wu);
        float os, ou;                   // and of that thread
        share(lane == first_lane, os, ou);
        if (lane == first_lane) waves[wave] = {m, ws, wu, os, ou, lane};
    }
    maxima[tid] = tmax;
    if (wave < 2 && lane < VEC) extras[wave * VEC + lane] = extra;
    __syncthreads();

    // ---- T -----------------------------------------------------------------------------------------------------------------------------
    // T: the smallest of the groups that fewer than K others exceed.  Each wavefront looks at 16 groups, four lanes each.
    if (a.top > 0) {
        float group = maxima[lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) group = fmaxf(group, maxima[lane + 64 * w]);
        groups[wave][lane] = group;
        const float mine = groups[wave][16 * wave + lane / 4];
        int above = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float o[4];
            __builtin_memcpy(o, &groups[wave][16 * (lane & 3) + 4 * j], 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) above += o[e] > mine ? 1 : 0;
        }
        above += __builtin_amdgcn_update_dpp(0, above, 0xB1, 0xF, 0xF, true);
        above += __builtin_amdgcn_update_dpp(0, above, 0x4E, 0xF, 0xF, true);
        const uint32_t least = wave_reduce(above < a.top ? ordered(mine) : ~0u, [](uint32_t p, uint32_t q) { return min(p, q); });
        if (lane == 0) atomicMin(&bound_bits, least);
    }
    // The workgroup's largest entry; wavefront 0 requests the entries of the first thread that has it, an entry a lane.
    float m = waves[0].m;
    int owner = 0;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
        owner = waves[w].m > m ? w : owner;
        m = fmaxf(m, waves[w].m);
    }
    const int owner_wave = owner;
    owner = 64 * owner + waves[owner].lane;
    const float far = m == -INFINITY ? 0.f : m;
    constexpr int SETS = (NV * VEC + 63) / 64;
    float owned[SETS + 1];
    if (wave == 0) {
#pragma unroll
        for (int k = 0; k < SETS; ++k) {
            const int e = k * 64 + lane, i = e / VEC * THREADS + owner;
            const float read = logit<T>(a.logits, first + (i < n_vecs ? id_of(i) + e % VEC : 0));
            owned[k] = i < n_vecs ? read : -INFINITY;
        }
        // (the thread's entry from in front or behind)
        owned[SETS] = lane == 0 && owner < 128 && (owner & 63) < VEC ? extras[(owner >> 6) * VEC + (owner & 63)] : -INFINITY;
    }
    __syncthreads();

    // ---- the vectors that may hold top entries, and their entries --------------------------------------------------------------------
    const float bound = unordered(bound_bits);
    if (a.top > 0) {
        const uint64_t below = (1ull << lane) - 1;
        int count = 0, equal = 0;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (v * THREADS >= n_vecs) continue;
            const bool in = v * THREADS + tid < n_vecs;
            if (__builtin_amdgcn_ballot_w64(in && vmax[v] >= bound) == 0) continue;
            const uint64_t eq = __builtin_amdgcn_ballot_w64(in && vmax[v] == bound);
            const bool take = in && (vmax[v] > bound || (vmax[v] == bound && equal + (int)__builtin_popcountll(eq & below) < a.top));
            const uint64_t taken = __builtin_amdgcn_ballot_w64(take);
            const int at = count + (int)__builtin_popcountll(taken & below);
            if (take && at < NEAR) near[wave][at] = v * THREADS + tid;
            count += (int)__builtin_popcountll(taken);
            equal += (int)__builtin_popcountll(eq);
        }
        auto offer = [&](bool in, float x, int id) {
            const bool take = in && x >= bound;
            const uint64_t taken = __builtin_amdgcn_ballot_w64(take);
            if (taken == 0) return;
            int at = 0;
            if (lane == 0) at = atomicAdd(&listed, (int)__builtin_popcountll(taken));
            at = __builtin_amdgcn_readfirstlane(at) + (int)__builtin_popcountll(taken & below);
            if (take && at < LIST) list[at] = key_of(x, id);
        };
        if (count > NEAR) {
            if (lane == 0) atomicAdd(&listed, LIST + 1);        // too many
        } else {
            for (int i = lane; i - lane < count * VEC; i += 64) {
                const int id = i < count * VEC ? id_of(near[wave][i / VEC]) + i % VEC : 0;
                offer(i < count * VEC, logit<T>(a.logits, first + id), id);
            }
        }
        offer(extra_id >= 0, extra, extra_id);
    }
    __syncthreads();
    // ---- sums: the owner's entries but one that is m, the threads that are their wavefront's first, all others ---------------------------
    if (wave == 0) {
        float S = 0.f, U = 0.f;
        bool out = false;
#pragma unroll
        for (int k = 0; k <= SETS; ++k) {
            const uint64_t is = __builtin_amdgcn_ballot_w64(owned[k] == m);
            const bool left_out = !out && is != 0 && lane == __builtin_ctzll(is);
            out = out || is != 0;
            const float y = fmaxf((owned[k] - far) * a.c, FAR), e = left_out ? 0.f : __builtin_amdgcn_exp2f(y);
            S += e;
            U = fmaf(y, e, U);
        }
        S = wave_sum(S);
        U = wave_sum(U);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const WaveSum x = waves[w];
            const float g = fmaxf((x.m - far) * a.c, FAR), f = x.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(g);
            const float ws = x.s + (w == owner_wave ? 0.f : x.os), wu = x.u + (w == owner_wave ? 0.f : x.ou);
            S += f * ws;
            U += f * fmaf(g, ws, wu);
        }
        if (ONE) {
            const RowSum r = row_sum(m, S, U);
            if (lane == 0) {
                sum = r;
                write_row<T>(a, row, r);
            }
        } else if (lane == 0) {
            a.parts[unit] = {m, S, U, 0.f};
        }
    }
    if (a.top == 0) return;
    auto put = [&](int place, uint64_t k) {
        if (ONE) write_top(a, row, place, k, sum);
        else a.keys[(size_t)unit * a.top + place] = k;
    };
    if (ONE) __syncthreads();
    const int all = listed;
    if (all > LIST) {
        uint64_t before = ~0ull;
        for (int place = 0; place < a.top; ++place) {
            uint64_t best = 0;
            auto look = [&](float x, int id) {
                const uint64_t k = key_of(x, id);
                if (k < before && k > best) best = k;
            };
            if (extra_id >= 0) look(extra, extra_id);
            for (int i = tid; i < n_vecs; i += THREADS) {
                float x[VEC];
                widen<T>(src[i], x);
#pragma unroll
                for (int j = 0; j < VEC; ++j) look(x[j], id_of(i) + j);
            }
            __syncthreads();                 // (of the round before, all have read the list)
            list[tid] = best;
            __syncthreads();
            for (int j = 0; j < THREADS; ++j) best = list[j] > best ? list[j] : best;
            if (tid == 0) put(place, best);
            before = best;
        }
        return;
    }
    for (int i = tid; i < all; i += THREADS) {
        const uint64_t k = list[i];
        int place = 0;
#pragma unroll 8
        for (int j = 0; j < all; ++j) place += list[j] > k ? 1 : 0;
        if (place < a.top) put(place, k);
    }
    // (fewer candidates than places: a short last piece, NaN)
    if (tid >= all && tid < a.top) put(tid, 0);
}

// sum over the wavefront, in every lane
__device__ __forceinline__ double wave_sum(double x)
{
    auto step = [&](auto move) {
        const uint64_t b = __builtin_bit_cast(uint64_t, x);
        const uint32_t lo = move((uint32_t)b), hi = move((uint32_t)(b >> 32));
        x += __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    };
    step([](uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true); });
    step([](uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true); });
    step([](uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true); });
    step([](uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true); });
    step([](uint32_t v) { return (uint32_t)__shfl_xor((int)v, 16); });
    step([](uint32_t v) { return (uint32_t)__shfl_xor((int)v, 32); });
    return x;
}

// The pieces of a row joined, sums in their order; one workgroup per row.  Latency is all it takes: what is read is requested at
// once, and the last wavefront works out the sums while the first ranks the top entries.
template <typename T>
__global__ __launch_bounds__(THREADS) void logprobs_join_kernel(Args a)
{
    const size_t row = wg_id_x();
    const int tid = thread_id_x(), lane = tid & 63, wave = tid >> 6;
    const Partial* const parts = a.parts + row * a.pieces;
    const uint64_t* const keys = a.keys + row * (size_t)a.pieces * a.top;
    const int batch = a.top > 0 ? 2 * THREADS / a.top : 1, all = min(a.pieces, batch) * a.top;     // pieces at a time, keys of the first ones
    __shared__ __align__(16) uint64_t list[2 * THREADS + MAX_TOP + 8];
    __shared__ uint64_t best[MAX_TOP], bound;
    __shared__ int listed;
    __shared__ RowSum sum;
    const uint8_t selected = a.mask ? a.mask[row] : 1;
    uint64_t mine[2] = {tid < all ? keys[tid] : 0, THREADS + tid < all ? keys[THREADS + tid] : 0};
    const Partial none = {-INFINITY, 0.f, 0.f, 0.f};
    Partial x = none;
    if (wave == WAVES - 1 && lane < a.pieces) x = parts[lane];
    if (selected != 1) return;

    auto sums = [&] {
        float m = x.m;
        for (int p = 64 + lane; p < a.pieces; p += 64) m = fmaxf(m, parts[p].m);
        m = wave_max(m);
        // the first piece that has the largest entry leaves it out
        int owner = 0x7fffffff;
        double s = 0.0, u = 0.0;
        for (int p0 = 0; p0 < a.pieces; p0 += 64) {
            const int p = p0 + lane;
            if (p0 > 0) x = p < a.pieces ? parts[p] : none;
            const uint64_t has = __builtin_amdgcn_ballot_w64(x.m == m);
            if (owner == 0x7fffffff && has) owner = p0 + __builtin_ctzll(has);
            if (x.m != -INFINITY) {
                const double d = ((double)x.m - (double)m) * a.c, f = x.m == m ? 1.0 : exp2(d), t = x.s + (p == owner ? 0.0 : 1.0);
                s += f * t;
                u += f * (x.u + d * t);
            }
        }
        const RowSum r = row_sum(m, wave_sum(s), wave_sum(u));
        if (lane == 0) {
            sum = r;
            write_row<T>(a, row, r);
        }
    };
    // The keys of as many pieces at a time as there is room for, with the best ones of the pieces before.  With n pieces and
    // t = ceil(top / n), the smallest of their t-th keys is one that n t >= top keys reach: only those from it on are ranked.
    if (tid < MAX_TOP) best[tid] = 0;
    for (int p0 = 0; p0 < a.pieces && a.top > 0; p0 += batch) {
        const int n = min(batch, a.pieces - p0), t = (a.top + n - 1) / n;
        if (tid == 0) {
            bound = ~0ull;
            listed = 0;
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i = h * THREADS + tid;
            if (p0 > 0) mine[h] = i < n * a.top ? keys[(size_t)p0 * a.top + i] : 0;
            if (i < n * a.top && i % a.top == t - 1) atomicMin(&bound, mine[h]);
        }
        __syncthreads();
        auto offer = [&](uint64_t k) {
            const uint64_t taken = __builtin_amdgcn_ballot_w64(k != 0 && k >= bound);
            if (taken == 0) return;
            int at = 0;
            if (lane == 0) at = atomicAdd(&listed, (int)__builtin_popcountll(taken));
            at = __builtin_amdgcn_readfirstlane(at) + (int)__builtin_popcountll(taken & ((1ull << lane) - 1));
            if (taken >> lane & 1) list[at] = k;
        };
        offer(mine[0]);
        offer(mine[1]);
        if (wave == 0) offer(lane < MAX_TOP ? best[lane] : 0);
        __syncthreads();
        const int m = listed;
        if (tid < 8) list[m + tid] = 0;
        __syncthreads();
        if (wave == WAVES - 1 && p0 + batch >= a.pieces) sums();      // (beside the ranks, which wavefront 0 mostly works out alone)
        for (int i = tid; i < m; i += THREADS) {
            const uint64_t k = list[i];
            int place = 0;
            for (int j = 0; j < m; j += 8)
#pragma unroll
                for (int e = 0; e < 8; ++e) place += list[j + e] > k ? 1 : 0;
            if (place < a.top) best[place] = k;
        }
        __syncthreads();
    }
    if (wave == WAVES - 1 && a.top == 0) sums();
    if (tid < a.top) write_top(a, row, tid, best[tid], sum);
}

struct LogprobPlan {
    int pieces, per;
    size_t parts_bytes, ws_bytes;
};

// A row that a workgroup can hold is one piece: one launch.  Others are cut into equal pieces, as few as hold them, or
// more where there are few rows: up to two workgroups a compute unit, of a quarter of what they can hold at least.  us with none
// finer, one, two, four, eight workgroups a compute unit: N=1, B=32, V=152064, top 5 12.4, 12.4, 11.7, 13.0, 13.6; V=50001, top 20 10.9, 10.1,
// 10.5, 10.5, 10.5; N=8, V=32768 12.5, 12.5, 12.4, 12.7, 13.9; pieces down to an eighth cost N=1, B=4 8 us (the join takes them in rounds).
LogprobPlan make_logprob_plan(const fdd_logprob_params& p)
{
    const long long vec = p.dtype == FDD_BF16 ? 8 : 4, rows = (long long)p.N * p.B;
    const long long vecs = std::max(p.V / vec, 1ll);            // (the entries in front of a row's first vector may take one from this)
    long long pieces = (vecs + MAX_NV * THREADS - 1) / (MAX_NV * THREADS);
    if (pieces > 1) {
        const long long finer = std::min(2ll * kNumCU / rows, (vecs + 2 * THREADS - 1) / (2 * THREADS));
        pieces = std::max(pieces, finer);
    }
    LogprobPlan l;
    l.per = (int)((vecs + pieces - 1) / pieces);
    l.pieces = (int)pieces;
    l.parts_bytes = pieces > 1 ? ((size_t)rows * pieces * sizeof(Partial) + 255) & ~(size_t)255 : 0;
    l.ws_bytes = pieces > 1 ? l.parts_bytes + (((size_t)rows * pieces * p.top * 8 + 255) & ~(size_t)255) : 0;
    return l;
}

}  // namespace

hipError_t launch_logprobs(const fdd_logprob_params& p, hipStream_t s)
{
    const LogprobPlan plan = make_logprob_plan(p);
    Args a;
    a.logits = p.logits;
    a.tokens = p.tokens;
    a.mask = p.row_mask;
    a.logprobs = p.logprobs;
    a.entropy = p.entropy;
    a.top = p.top_ids ? p.top : 0;
    a.top_ids = p.top_ids;
    a.top_logprobs = p.top_logprobs;
    a.parts = static_cast<Partial*>(p.workspace);
    a.keys = reinterpret_cast<uint64_t*>(static_cast<char*>(p.workspace) + plan.parts_bytes);
    a.V = p.V;
    a.rows = p.N * p.B;
    a.pieces = plan.pieces;
    a.per = plan.per;
    a.dPieces = make_fastdiv((uint32_t)plan.pieces);
    a.inv_t = 1.f / p.temperature;
    a.c = LOG2E * a.inv_t;
    const dim3 rows((unsigned)a.rows), units((unsigned)a.rows * (unsigned)plan.pieces), block(THREADS);
    const bool bf16 = p.dtype == FDD_BF16, one = plan.pieces == 1, compact = a.mask && a.rows >= 16 && a.rows <= LIVE_ROWS;   // (as many as eligible_row takes; N=8, B=32, half of the rows: 18.9 us, else 21.1)
    auto held = [&](auto is_one, auto is_compact, auto nv) {
        constexpr bool ONE = decltype(is_one)::value, COMPACT = decltype(is_compact)::value;
        constexpr int NV = decltype(nv)::value;
        if (bf16) hipLaunchKernelGGL((logprobs_kernel<uint16_t, ONE, COMPACT, NV>), units, block, 0, s, a);
        else hipLaunchKernelGGL((logprobs_kernel<float, ONE, COMPACT, NV>), units, block, 0, s, a);
    };
    auto go = [&](auto is_one, auto is_compact) {
        if (plan.per <= FEW_NV * THREADS) held(is_one, is_compact, std::integral_constant<int, FEW_NV>());
        else held(is_one, is_compact, std::integral_constant<int, MAX_NV>());
    };
    if (one && compact) go(std::true_type(), std::true_type());
    else if (one) go(std::true_type(), std::false_type());
    else if (compact) go(std::false_type(), std::true_type());
    else go(std::false_type(), std::false_type());
    if (hipError_t e = hipGetLastError(); e != hipSuccess || one) return e;
    if (bf16) hipLaunchKernelGGL(logprobs_join_kernel<uint16_t>, rows, block, 0, s, a);
    else hipLaunchKernelGGL(logprobs_join_kernel<float>, rows, block, 0, s, a);
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
    // a launch takes less than 2^32 work items
    if ((long long)p->N * p->B * make_logprob_plan(*p).pieces > (1ll << 23)) return fail(FDD_ERR_SHAPE, "%s: N*B*V too large", fn);
    return FDD_OK;
}

extern "C" {

size_t fdd_token_logprobs_workspace(const fdd_logprob_params* p)
{
    if (check_shape(p, "fdd_token_logprobs_workspace") != FDD_OK) return 0;
    return make_logprob_plan(*p).ws_bytes;
}

fdd_status fdd_token_logprobs(const fdd_logprob_params* p)
{
    const char* const fn = "fdd_token_logprobs";
    fdd_status st = check_shape(p, fn);
    if (st != FDD_OK) return st;
    // (0 log2(e) / temperature has to be 0; and a difference of logits that fp32 cannot hold, 2^128 and more, has to be one whose exponential
    // is 0: its y is 2^128 log2(e) / 2^120 = 369 below the largest at least, beyond FAR)
    if (!(p->temperature > 0.f) || p->temperature > 0x1p120f || std::isinf(1.5f / p->temperature))
        return fail(FDD_ERR_UNSUPPORTED, "%s: temperature must be positive and at most 2^120, and 1.5 / temperature finite", fn);
    if (!p->logits) return fail(FDD_ERR_NULL, "%s: logits must not be NULL", fn);
    if (p->logprobs && !p->tokens) return fail(FDD_ERR_NULL, "%s: logprobs need tokens", fn);
    if (p->top > 0 && !p->top_ids != !p->top_logprobs) return fail(FDD_ERR_NULL, "%s: top_ids and top_logprobs come together", fn);
    if (!p->logprobs && !p->entropy && !(p->top > 0 && p->top_ids)) return fail(FDD_ERR_NULL, "%s: no output to compute", fn);
    if (reinterpret_cast<uintptr_t>(p->logits) & 15u) return fail(FDD_ERR_UNSUPPORTED, "%s: logits must be 16-byte aligned", fn);
    const void* words[] = {p->tokens, p->logprobs, p->entropy, p->top_ids, p->top_logprobs};
    for (const void* w : words)
        if (reinterpret_cast<uintptr_t>(w) & 3u) return fail(FDD_ERR_UNSUPPORTED, "%s: tokens and outputs must be 4-byte aligned", fn);
    const size_t need = make_logprob_plan(*p).ws_bytes;
    if (need > 0) {
        if (!p->workspace) return fail(FDD_ERR_WORKSPACE, "%s: workspace is NULL, %zu bytes needed", fn, need);
        if (reinterpret_cast<uintptr_t>(p->workspace) & 255u) return fail(FDD_ERR_WORKSPACE, "%s: workspace must be 256-byte aligned", fn);
        if (p->workspace_bytes < need) return fail(FDD_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", fn, p->workspace_bytes, need);
    }
    hipError_t e = launch_logprobs(*p, static_cast<hipStream_t>(p->stream));
    if (e != hipSuccess) return fail(FDD_ERR_LAUNCH, "%s: launch failed: %s", fn, hipGetErrorString(e));
    return FDD_OK;
}

}  // extern "C"
