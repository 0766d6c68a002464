// Which drafted tokens of a tree or a chain stand, from given random numbers (fdd_tree_verify).
//
// With p the target's distribution behind a token and q the one a child was drawn from (or 1, where it was chosen), a child x
// stands with probability min(1, p(x) / q(x)), and what is drawn where none does comes from what q leaves of p, max(p - q, 0) (or
// from p without the children): token after token is then distributed as p.
//
// Four launches (two where the target is greedy):
//   stats   one read of the logits: maximum and sum of exponentials of pieces of every row that is there
//   walk    one workgroup per request: joins the pieces, tests the children, leaves the path and the token it ends at
//   weigh   the row of that token alone, once more and in fp64: sums of pieces of what the last token is drawn from
//           (a chain with draft_logits: both rows' sums, and in a launch behind it those of max(p - q, 0))
//   pick    the piece that the uniform falls into, entry by entry
// stats is bound by bytes, what is behind it by the latency of its launches and of the steps that depend on one another: 8 trees of 32 tokens,
// V = 152064 in bf16, 33.1 us = stats 17.0 (4.6 TB/s), walk 6.3, weigh 5.3, pick 6.1, less what they overlap; 4 chains of 9 tokens, V = 50001 in
// fp32 with draft_logits, 27.2 us = stats 6.0, walk 4.8, weigh 5.2 and 4.9, pick 6.1.  Greedy, from a graph: the same trees 19.6 us, the chains 8.4.
// (walk in every workgroup of weigh, a launch less: 8 trees of 32 tokens 33.0 -> 31.0 us, but one of 16, V = 152064, 18.4 -> 20.8 and 2 of 200, V = 50001,
// 29.5 -> 32.5, as they were then: not kept.)
// A test compares a probability with what the children that fell have left of the row.  stats takes fp32 exponentials and adds them in fp64, the
// tokens' own exponentials and all that walk does with them are fp64: a probability is off by what the row's sum is, 2^-16 of itself at
// most, however small it is.  (An entry a octaves below the reference has an exponent of three roundings, 3 ln2 a 2^-24 of the entry, and a
// row's entries are log2 V octaves below on average, their weights counted, at most; 2^-22.4 for the sums of 8, 2^-23 for the exponential and for each time
// that the reference moves, by 8 octaves and more in a thread; then the threads', wavefronts' and pieces' references, whose distances add up once more.)
// What is left, one less the probabilities that fell, is off by 2^-16 of what fell.
// The draw compares with V borders that lie as close as the smallest probabilities: an fp32 exponential's error, summed over the row, would move one draw in a
// few hundred (V = 152064, logits of deviation 2) to a neighbouring entry, so these exponentials are fp64 too, and only one row a request needs them.
#include <cfloat>

#include "paged.h"
#include "wave.h"

namespace fdd {
namespace tree_verify {

constexpr int MAX_PIECES = 64;          // a wavefront joins a row's
constexpr int STAT_THREADS = 256, WALK_THREADS = 1024;
constexpr int WP = 1024, PICK = 8;      // pieces of the row that is drawn from, at most; its entries that a thread looks at together
constexpr double LOG2E = 1.4426950408889634074;
constexpr double NOTHING_LEFT = 0x1p-40;

struct Stat {        // of a piece of a row
    float max;       // (not greedy: the reference, up to 8 octaves of the exponentials below the largest)
    int arg;         // greedy: lowest id of the largest
    double sum;      // of exp((x - max) / temperature)
};

// per request, from `walk` to the launches behind it
struct Stop {
    int token;              // where the walk ended, or -1: nothing to draw
    int n_path;
    float max, draft_max;   // of the two rows
    int children;           // entries of the request's list: ids of the children that fell
    int residue;            // a chain with draft_logits whose next token fell
};

struct Args {
    const void* logits;
    const void* draft;
    const int32_t* tokens;
    const int32_t* parents;
    long long parents_stride;
    const float* uniforms;
    const int32_t* n_tokens;
    int32_t* path;
    int32_t* n_path;
    int32_t* emitted;
    float* chances;
    Stat* stats;            // [2][N*B][pieces]
    Stop* stops;            // [N]
    int32_t* lists;         // [N,B]
    double* sums;           // [3][N][w_pieces]: of p, of what is drawn from, of q
    int N, B, V, pieces, per_piece;       // per_piece: entries, a multiple of 8
    int w_pieces, w_per;                  // of the row that is drawn from
    float c, draft_c;                     // log2(e) / temperature
    float slack, draft_slack;             // 8 octaves
    double c64, draft_c64;
};

__device__ __forceinline__ int count_of(const Args& a, int n) { return a.n_tokens ? min(max(a.n_tokens[n], 0), a.B) : a.B; }
__device__ __forceinline__ int parent_at(const Args& a, int n, int j)
{
    if (j == 0) return -1;
    return a.parents ? parent_of(j, a.parents[n * a.parents_stride + j]) : j - 1;
}

template <typename T>
__device__ __forceinline__ float entry(const T* p)
{
    if constexpr (sizeof(T) == 2) return __builtin_bit_cast(float, (uint32_t)*p << 16);
    else return *p;
}
// 16 bytes of a row, which may start anywhere
template <typename T>
__device__ __forceinline__ void entries(const T* p, float (&x)[16 / sizeof(T)])
{
    uint32_t w[4];
    __builtin_memcpy(w, p, 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2) {
            x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
            x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
        } else {
            x[i] = __builtin_bit_cast(float, w[i]);
        }
    }
}

__device__ __forceinline__ double exponential(float x, double top, double c) { return exp2(((double)x - top) * c); }

__device__ __forceinline__ double wave_sum(double x)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    return x;
}

// ---- stats -------------------------------------------------------------------------------------------------------------
template <typename T, bool GREEDY>
__global__ __launch_bounds__(STAT_THREADS) void stats_kernel(Args a)
{
    constexpr int VE = 16 / sizeof(T);
    __shared__ float s_max[STAT_THREADS / 64];
    __shared__ double s_sum[STAT_THREADS / 64];
    __shared__ int s_arg[STAT_THREADS / 64];
    const int piece = blockIdx.x % a.pieces, row = blockIdx.x / a.pieces, which = blockIdx.y;
    const int n = row / a.B, i = row - n * a.B;
    const int count = count_of(a, n);
    if (i >= count || (which && i + 1 >= count)) return;       // (a draft's last row has no token behind it)
    const T* const x = static_cast<const T*>(which ? a.draft : a.logits) + (long long)row * a.V;
    const float c = which ? a.draft_c : a.c, slack = which ? a.draft_slack : a.slack;
    const int v0 = piece * a.per_piece, v1 = min(v0 + a.per_piece, a.V);
    float m = -FLT_MAX;          // (never above the entries, but for -inf, which weighs nothing)
    double s = 0.0;
    int arg = v0;
    bool any = false;
    auto take = [&](const float* y, int count_y, int v) {
        float best = y[0];
        int at = 0;
        for (int j = 1; j < count_y; ++j)
            if (y[j] > best) {
                best = y[j];
                at = j;
            }
        if constexpr (GREEDY) {
            if (!any || best > m) {
                m = best;
                arg = v + at;
                any = true;
            }
        } else {
            if (best > m + slack) {       // (rarely: each time rounds the sum)
                s *= (double)__builtin_amdgcn_exp2f((m - best) * c);
                m = best;
            }
            float few = 0.f;
            for (int j = 0; j < count_y; ++j) few += __builtin_amdgcn_exp2f((y[j] - m) * c);
            s += (double)few;
        }
    };
    const int whole = v0 + (v1 - v0) / VE * VE;
    for (int v = v0 + threadIdx.x * VE; v < whole; v += STAT_THREADS * VE) {
        float y[VE];
        entries(x + v, y);
        take(y, VE, v);
    }
    if (whole + (int)threadIdx.x < v1) {
        const float y = entry(x + whole + threadIdx.x);
        take(&y, 1, whole + threadIdx.x);
    }
    if (GREEDY && !any) m = -INFINITY, arg = a.V;          // (a thread without entries)
    // join the threads
    for (int d = 1; d < 64; d *= 2) {
        const float m2 = __shfl_xor(m, d);
        const int arg2 = __shfl_xor(arg, d);
        if constexpr (GREEDY) {
            if (m2 > m || (m2 == m && arg2 < arg)) m = m2, arg = arg2;
        } else {
            const double s2 = __shfl_xor(s, d);
            const float top = fmaxf(m, m2);
            s = s * (double)__builtin_amdgcn_exp2f((m - top) * c) + s2 * (double)__builtin_amdgcn_exp2f((m2 - top) * c);
            m = top;
        }
    }
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) s_max[wave] = m, s_sum[wave] = s, s_arg[wave] = arg;
    __syncthreads();
    if (threadIdx.x) return;
    double sum = 0.0;
    for (int w = 0; w < STAT_THREADS / 64; ++w)
        if (GREEDY ? s_max[w] > m || (s_max[w] == m && s_arg[w] < arg) : s_max[w] > m) m = s_max[w], arg = s_arg[w];
    for (int w = 0; w < STAT_THREADS / 64; ++w) sum += s_sum[w] * (double)__builtin_amdgcn_exp2f((s_max[w] - m) * c);
    Stat r;
    r.max = m;
    r.arg = min(arg, a.V - 1);
    r.sum = GREEDY ? 0.0 : sum;
    a.stats[((long long)which * a.N * a.B + row) * a.pieces + piece] = r;
}

// ---- walk --------------------------------------------------------------------------------------------------------------
// Bound by the latency of what depends on one another: lists, then pieces and the tokens' logits, then LDS only.
template <typename T, bool GREEDY>
__global__ __launch_bounds__(WALK_THREADS) void walk_kernel(Args a)
{
    __shared__ float s_max[2][FDD_TREE_MAX];
    __shared__ double s_sum[2][FDD_TREE_MAX];
    __shared__ int s_arg[FDD_TREE_MAX], s_token[FDD_TREE_MAX], s_parent[FDD_TREE_MAX];
    __shared__ double s_p[FDD_TREE_MAX], s_q[FDD_TREE_MAX];      // of a token, under its parent's rows
    __shared__ float s_u[FDD_TREE_MAX];
    const int n = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool draft = !GREEDY && a.draft;
    const long long row0 = (long long)n * a.B;
    // a thread has one token (B <= WALK_THREADS)
    const int j = tid, jc = min(j, a.B - 1);
    const int token = a.tokens[row0 + jc];
    const int parent = parent_at(a, n, jc);
    const float u = GREEDY ? 0.f : a.uniforms[(row0 + jc) * 2];
    const int count = count_of(a, n);
    const bool there = j < count, inside = token >= 0 && token < a.V;
    float of_p = 0.f, of_q = 0.f;
    if (!GREEDY && there && parent >= 0 && inside) {
        of_p = entry(static_cast<const T*>(a.logits) + (row0 + parent) * a.V + token);
        if (draft) of_q = entry(static_cast<const T*>(a.draft) + (row0 + parent) * a.V + token);
    }
    // rows: a power of two of lanes joins the pieces of one
    int span = 1;
    while (span < a.pieces) span *= 2;
    for (int r0 = wave * (64 / span); r0 < (draft ? 2 : 1) * count; r0 += WALK_THREADS / span) {
        const int r = r0 + lane / span, piece = lane & (span - 1);
        const int which = r >= count, i = which ? r - count : r;
        const bool row = r < (draft ? 2 : 1) * count && !(which && i + 1 >= count);
        const float c = which ? a.draft_c : a.c;
        Stat st = {-INFINITY, a.V - 1, 0.0};
        if (row && piece < a.pieces) st = a.stats[((long long)which * a.N * a.B + row0 + i) * a.pieces + piece];
        float m = st.max;
        int arg = st.arg;
        for (int d = 1; d < span; d *= 2) {
            const float m2 = __shfl_xor(m, d);
            const int arg2 = __shfl_xor(arg, d);
            if (m2 > m || (m2 == m && arg2 < arg)) m = m2, arg = arg2;
        }
        double sum = GREEDY || !row || piece >= a.pieces ? 0.0 : st.sum * (double)__builtin_amdgcn_exp2f((st.max - m) * c);
        if (!GREEDY)
            for (int d = 1; d < span; d *= 2) sum += __shfl_xor(sum, d);
        if (row && piece == 0) {
            s_max[which][i] = m;
            s_sum[which][i] = sum;
            if (GREEDY) s_arg[i] = arg;
        }
    }
    if (j < a.B) {
        s_parent[j] = there ? parent : -1;
        s_token[j] = token;
        s_u[j] = u;
    }
    __syncthreads();
    if (j < a.B) {
        double p = 0.0, q = 1.0, chance = there && j == 0 ? 1.0 : 0.0;
        if (there && parent >= 0 && inside) {
            if constexpr (GREEDY) {
                p = token == s_arg[parent] ? 1.0 : 0.0;
            } else {
                p = exponential(of_p, s_max[0][parent], a.c64) / s_sum[0][parent];
                if (draft) q = exponential(of_q, s_max[1][parent], a.draft_c64) / s_sum[1][parent];
            }
            chance = draft && q > 0.0 ? fmin(1.0, p / q) : draft && p > 0.0 ? 1.0 : fmin(1.0, p);
        }
        if (a.chances) a.chances[row0 + j] = (float)chance;
        // a token that an earlier child of the same parent has is no longer there when it is tried
        bool again = false;
        if (!draft && !GREEDY && there && parent >= 0)
            for (int i = parent + 1; i < j; ++i) again = again || (s_parent[i] == parent && s_token[i] == token);
        s_p[j] = again ? 0.0 : p;
        s_q[j] = q;
    }
    __syncthreads();
    if (wave) return;
    // children have higher numbers than their parent and are tried in order, so one pass over the tokens meets all of them
    int now = 0, steps = 0;        // (uniform)
    double left = 1.0;             // of p, behind the children that fell
    for (int j0 = 0; j0 < count; j0 += 64) {
        const int k = j0 + lane;
        const bool here = k > 0 && k < count;
        const int up = here ? s_parent[k] : -1, x = here ? s_token[k] : -1;
        const double p = here ? s_p[k] : 0.0, uq = here ? (double)s_u[k] * s_q[k] : 0.0;
        int from = j0;
        for (;;) {
            const uint64_t tried = __builtin_amdgcn_ballot_w64(here && up == now && k >= from);
            if (tried == 0) break;
            const int l = __builtin_ctzll(tried);
            auto of = [&](double y) { return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(y), l), __builtin_amdgcn_readlane(__double2loint(y), l)); };
            const double p_l = of(p), uq_l = of(uq);
            from = j0 + l + 1;
            const bool stands = GREEDY ? p_l > 0.0 : uq_l * left < p_l;
            if (stands) {
                now = j0 + l;
                if (lane == l) {
                    a.emitted[row0 + steps] = x;
                    a.path[row0 + steps + 1] = k;
                }
                ++steps;
                left = 1.0;
            } else {
                left -= p_l;
            }
        }
    }
    // (each entry has one writer: this wavefront, and for the token drawn last the last launch)
    for (int k = lane; k < a.B; k += 64) {
        if (count == 0 || k > steps) a.path[row0 + k] = a.emitted[row0 + k] = -1;
        else if (k == 0) a.path[row0] = 0;
    }
    int children = 0;
    if (!GREEDY && !draft)
        for (int j0 = now & ~63; j0 < count; j0 += 64) {
            const int k = j0 + lane;
            const bool child = k > now && k < count && s_parent[k] == now;
            const uint64_t all = __builtin_amdgcn_ballot_w64(child);
            if (child) a.lists[row0 + children + __builtin_popcountll(all & ((1ull << lane) - 1))] = s_token[k];
            children += __builtin_popcountll(all);
        }
    if (lane == 0) {
        a.n_path[n] = count > 0 ? steps + 1 : 0;
        if constexpr (GREEDY) {
            if (count > 0) a.emitted[row0 + steps] = s_arg[now];
        } else {
            Stop st;
            st.token = count > 0 ? now : -1;
            st.n_path = steps + 1;
            st.max = count > 0 ? s_max[0][now] : 0.f;
            st.residue = draft && now + 1 < count;
            st.draft_max = st.residue ? s_max[1][now] : 0.f;
            st.children = children;
            a.stops[n] = st;
        }
    }
}

// ---- weigh -------------------------------------------------------------------------------------------------------------
// What the last token is drawn from: p without the children of the token where the walk ended; or max(p - q, 0) where a chain's next
// token fell.  A thread has PICK entries that follow one another.
template <typename T>
struct Weights {
    const T* p;
    const T* q;
    int V, children;
    const int* list;            // in LDS
    bool residue;
    double p_max, q_max, p_c, q_c, p_scale, q_scale;

    __device__ __forceinline__ Weights(const Args& a, int n, const Stop& st, const int* children_ids)
    {
        const long long row = ((long long)n * a.B + st.token) * a.V;
        p = static_cast<const T*>(a.logits) + row;
        residue = st.residue != 0;
        q = residue ? static_cast<const T*>(a.draft) + row : nullptr;
        V = a.V;
        children = st.children;
        list = children_ids;
        p_max = st.max;
        q_max = st.draft_max;
        p_c = a.c64;
        q_c = a.draft_c64;
        p_scale = q_scale = 1.0;
    }
    __device__ __forceinline__ void read(const T* row, int v, float (&x)[PICK]) const
    {
        constexpr int VE = 16 / sizeof(T);
        if (v + PICK <= V) {
            float y[PICK / VE][VE];
#pragma unroll
            for (int i = 0; i < PICK / VE; ++i) entries(row + v + i * VE, y[i]);
#pragma unroll
            for (int i = 0; i < PICK; ++i) x[i] = y[i / VE][i % VE];
        } else {
#pragma unroll
            for (int i = 0; i < PICK; ++i) x[i] = v + i < V ? entry(row + v + i) : -INFINITY;
        }
    }
    // bits of the entries at v that were children's
    __device__ __forceinline__ uint32_t taken(int v) const
    {
        uint32_t bits = 0;
        for (int i = 0; i < children; ++i) {
            const uint32_t d = (uint32_t)(list[i] - v);
            bits |= d < (uint32_t)PICK ? 1u << d : 0u;
        }
        return bits;
    }
};
// the request's stop and its children's ids, in LDS
__device__ __forceinline__ Stop get_stop(const Args& a, int n, int* list)
{
    const Stop st = a.stops[n];
    if (!a.draft)
        for (int i = threadIdx.x; i < a.B; i += STAT_THREADS) list[i] = a.lists[(long long)n * a.B + i];      // (those behind the last are not used)
    __syncthreads();
    return st;
}
__device__ __forceinline__ double wg_sum(double x, double* scratch)
{
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = x;
    __syncthreads();
    double s = 0.0;
    for (int w = 0; w < STAT_THREADS / 64; ++w) s += scratch[w];
    return s;
}
// sum of the threads before this one
__device__ __forceinline__ double wg_before(double x, double* scratch)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double end = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const double y = __shfl_up(end, d);
        if (lane >= d) end += y;
    }
    __syncthreads();
    if (lane == 63) scratch[wave] = end;
    __syncthreads();
    double before = __shfl_up(end, 1);
    if (lane == 0) before = 0.0;
    for (int w = 0; w < STAT_THREADS / 64; ++w) before += w < wave ? scratch[w] : 0.0;
    return before;
}
// lowest of the threads' first and highest of their second numbers.  (Of LDS atomics to one place the compiler makes a loop over the lanes:
// two of them for each entry were 35 us of a call.)
__device__ __forceinline__ void wg_first_last(int* first, int* last, int* scratch)
{
    const int f = (int)wave_reduce((uint32_t)*first, [](uint32_t x, uint32_t y) { return (uint32_t)min((int)x, (int)y); });
    const int l = (int)wave_reduce((uint32_t)*last, [](uint32_t x, uint32_t y) { return (uint32_t)max((int)x, (int)y); });
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        scratch[threadIdx.x >> 6] = f;
        scratch[STAT_THREADS / 64 + (threadIdx.x >> 6)] = l;
    }
    __syncthreads();
    *first = scratch[0];
    *last = scratch[STAT_THREADS / 64];
    for (int w = 1; w < STAT_THREADS / 64; ++w) {
        *first = min(*first, scratch[w]);
        *last = max(*last, scratch[STAT_THREADS / 64 + w]);
    }
}
// Sum of a row's pieces, in every lane.  (Every wavefront for itself: no barrier.  So is the search below.)
__device__ __forceinline__ double row_sum(const double* sums, int n)
{
    double s = 0.0;
    for (int i = threadIdx.x & 63; i < n; i += 64) s += sums[i];
    return wave_sum(s);
}
// The piece that `share` of the sum of all falls into, the first whose end lies above it, or (by rounding) the last one with any
// weight, and what of the sum lies in front of it; lane l has pieces l each .. (l + 1) each - 1.
struct Found {
    int piece;
    double target, before;
};
__device__ __forceinline__ Found find_piece(const double* sums, int n, double share)
{
    const int lane = threadIdx.x & 63, each = (n + 63) >> 6, first = lane * each;
    double mine = 0.0;
    for (int i = 0; i < each; ++i) mine += first + i < n ? sums[first + i] : 0.0;
    double end = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const double y = __shfl_up(end, d);
        if (lane >= d) end += y;
    }
    Found f;
    f.target = share * __shfl(end, 63);
    const uint64_t over = __builtin_amdgcn_ballot_w64(mine > 0.0 && end > f.target), any = __builtin_amdgcn_ballot_w64(mine > 0.0);
    const int l = over ? __builtin_ctzll(over) : any ? 63 - __builtin_clzll(any) : 0;
    double at = __shfl(end - mine, l);
    f.piece = min(l * each, n - 1);
    f.before = at;
    for (int i = 0; i < each && l * each + i < n; ++i) {
        const double s = sums[l * each + i];
        if (s > 0.0) {
            f.piece = l * each + i;
            f.before = at;
            if (at + s > f.target) break;
        }
        at += s;
    }
    return f;
}

template <typename T, bool RESIDUE>
__global__ __launch_bounds__(STAT_THREADS) void weigh_kernel(Args a)
{
    __shared__ int list[FDD_TREE_MAX];
    __shared__ double scratch[STAT_THREADS / 64];
    const int piece = blockIdx.x % a.w_pieces, n = blockIdx.x / a.w_pieces;
    const long long np = (long long)a.N * a.w_pieces, at = (long long)n * a.w_pieces + piece;
    const Stop st = get_stop(a, n, list);
    if (st.token < 0 || (RESIDUE && !st.residue)) return;
    Weights<T> w(a, n, st, list);
    const int v0 = piece * a.w_per, v1 = min(v0 + a.w_per, a.V);
    double all = 0.0, left = 0.0, other = 0.0;
    if constexpr (RESIDUE) {
        w.p_scale = 1.0 / row_sum(a.sums + (long long)n * a.w_pieces, a.w_pieces);
        w.q_scale = 1.0 / row_sum(a.sums + 2 * np + (long long)n * a.w_pieces, a.w_pieces);
    }
    for (int v = v0 + threadIdx.x * PICK; v < v1; v += STAT_THREADS * PICK) {
        float x[PICK], y[PICK];
        w.read(w.p, v, x);
        if (w.residue) w.read(w.q, v, y);
        if constexpr (RESIDUE) {
#pragma unroll
            for (int i = 0; i < PICK; ++i) left += fmax(exponential(x[i], w.p_max, w.p_c) * w.p_scale - exponential(y[i], w.q_max, w.q_c) * w.q_scale, 0.0);
        } else {
            const uint32_t taken = w.taken(v);
#pragma unroll
            for (int i = 0; i < PICK; ++i) {
                const double e = exponential(x[i], w.p_max, w.p_c);
                all += e;
                left += taken >> i & 1 ? 0.0 : e;
                if (w.residue) other += exponential(y[i], w.q_max, w.q_c);
            }
        }
    }
    left = wg_sum(left, scratch);
    if constexpr (!RESIDUE) {
        all = wg_sum(all, scratch);
        if (w.residue) other = wg_sum(other, scratch);
    }
    if (threadIdx.x == 0) {
        a.sums[np + at] = left;
        if constexpr (!RESIDUE) {
            a.sums[at] = all;
            if (w.residue) a.sums[2 * np + at] = other;
        }
    }
}

// ---- pick --------------------------------------------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(STAT_THREADS) void pick_kernel(Args a)
{
    __shared__ int list[FDD_TREE_MAX];
    __shared__ int ends[2 * STAT_THREADS / 64];
    __shared__ double scratch[STAT_THREADS / 64];
    const int n = blockIdx.x, tid = threadIdx.x;
    const long long np = (long long)a.N * a.w_pieces;
    const double* const p_sums = a.sums + (long long)n * a.w_pieces;
    const Stop st = get_stop(a, n, list);
    if (st.token < 0) return;
    Weights<T> w(a, n, st, list);
    const float u = a.uniforms[((long long)n * a.B + st.token) * 2 + 1];
    const double* sums = p_sums + np;
    const double all = row_sum(p_sums, a.w_pieces), total = row_sum(sums, a.w_pieces);
    if (w.residue) {
        w.p_scale = 1.0 / all;
        w.q_scale = 1.0 / row_sum(p_sums + 2 * np, a.w_pieces);
    }
    if (total < NOTHING_LEFT * (w.residue ? 1.0 : all)) {       // the drafts account for all of p
        w.residue = false;
        w.children = 0;
        sums = p_sums;
    }
    const Found f = find_piece(sums, a.w_pieces, (double)u);
    double left = f.target - f.before;
    int first, last = -1;
    // its entries, STAT_THREADS * PICK at a time
    const int v0 = f.piece * a.w_per, v1 = min(v0 + a.w_per, a.V);
    first = INT32_MAX;
    for (int b = v0; b < v1; b += STAT_THREADS * PICK) {
        const int v = b + tid * PICK;
        double x[PICK], sum = 0.0;
        if (v < v1) {
            float p[PICK], q[PICK];
            w.read(w.p, v, p);
            if (w.residue) w.read(w.q, v, q);
            const uint32_t taken = w.residue ? 0u : w.taken(v);
#pragma unroll
            for (int i = 0; i < PICK; ++i) {
                const double e = exponential(p[i], w.p_max, w.p_c);
                x[i] = w.residue ? fmax(e * w.p_scale - exponential(q[i], w.q_max, w.q_c) * w.q_scale, 0.0) : taken >> i & 1 ? 0.0 : e;
            }
        } else {
#pragma unroll
            for (int i = 0; i < PICK; ++i) x[i] = 0.0;
        }
#pragma unroll
        for (int i = 0; i < PICK; ++i) sum += x[i];
        double end = wg_before(sum, scratch);
        int from = INT32_MAX, to = last;
#pragma unroll
        for (int i = 0; i < PICK; ++i) {
            end += x[i];
            if (!(x[i] > 0.0)) continue;
            to = b + tid * PICK + i;
            if (end > left) from = min(from, to);
        }
        wg_first_last(&from, &to, ends);
        first = from;
        last = to;
        if (first != INT32_MAX) break;
        left -= wg_sum(sum, scratch);
    }
    if (tid == 0) a.emitted[(long long)n * a.B + st.n_path - 1] = first != INT32_MAX ? first : last >= 0 ? last : v0;
}

// ---- host ----------------------------------------------------------------------------------------------------------------

struct Plan {
    int pieces, per_piece, w_pieces, w_per;
    size_t stats, stops, lists, sums;      // bytes
};

Plan make_plan(const fdd_tree_verify_params& p)
{
    const long long rows = (long long)p.N * p.B * (p.draft_logits ? 2 : 1);
    long long pieces = (8ll * kNumCU + rows - 1) / rows;
    const long long most = (p.V + 2047) / 2048;
    if (pieces > most) pieces = most;
    if (pieces > MAX_PIECES) pieces = MAX_PIECES;
    if (pieces < 1) pieces = 1;
    Plan pl;
    pl.per_piece = (int)(((p.V + pieces - 1) / pieces + 7) / 8 * 8);
    pl.pieces = (int)((p.V + pl.per_piece - 1) / pl.per_piece);
    auto round = [](size_t x) { return (x + 255) & ~(size_t)255; };
    pl.stats = round((size_t)rows * pl.pieces * sizeof(Stat));
    pl.stops = round((size_t)p.N * sizeof(Stop));
    pl.lists = round((size_t)p.N * p.B * sizeof(int32_t));
    constexpr int unit = STAT_THREADS * PICK;
    pl.w_per = (int)(((p.V + WP - 1) / WP + unit - 1) / unit * unit);
    pl.w_pieces = (int)((p.V + pl.w_per - 1) / pl.w_per);
    pl.sums = round((size_t)3 * p.N * pl.w_pieces * sizeof(double));
    return pl;
}

template <typename T>
hipError_t launch(const Args& a, bool greedy, hipStream_t s)
{
    const dim3 stats((unsigned)((long long)a.N * a.B * a.pieces), a.draft ? 2u : 1u);
    if (greedy) {
        stats_kernel<T, true><<<stats, STAT_THREADS, 0, s>>>(a);
        walk_kernel<T, true><<<dim3((unsigned)a.N), WALK_THREADS, 0, s>>>(a);
        return hipGetLastError();
    }
    const dim3 rows((unsigned)((long long)a.N * a.w_pieces));
    stats_kernel<T, false><<<stats, STAT_THREADS, 0, s>>>(a);
    walk_kernel<T, false><<<dim3((unsigned)a.N), WALK_THREADS, 0, s>>>(a);
    weigh_kernel<T, false><<<rows, STAT_THREADS, 0, s>>>(a);
    if (a.draft) weigh_kernel<T, true><<<rows, STAT_THREADS, 0, s>>>(a);
    pick_kernel<T><<<dim3((unsigned)a.N), STAT_THREADS, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace tree_verify
}  // namespace fdd

using namespace fdd;
using namespace fdd::tree_verify;

#define fail set_error

namespace {

const char* const kFn = "fdd_tree_verify";

bool in_range(float t) { return t >= 0x1p-20f && t <= 0x1p20f; }

fdd_status check_shape(const fdd_tree_verify_params* p)
{
    if (!p) return fail(FDD_ERR_NULL, "%s: params is NULL", kFn);
    if (p->N <= 0 || p->B <= 0 || p->V <= 0) return fail(FDD_ERR_SHAPE, "%s: N, B, V must be positive (got N=%d B=%d V=%lld)", kFn, p->N, p->B, (long long)p->V);
    if (p->B > FDD_TREE_MAX) return fail(FDD_ERR_UNSUPPORTED, "%s: B=%d is above %d", kFn, p->B, FDD_TREE_MAX);
    if (p->V > (1ll << 30)) return fail(FDD_ERR_SHAPE, "%s: V must be at most 2^30", kFn);
    // (a launch has at most 2^32 threads: 256 for each piece of a row, 1024 for a request)
    if (p->N >= (1 << 22) || (long long)p->N * p->B >= (1ll << 24)) return fail(FDD_ERR_SHAPE, "%s: N or N*B too large", kFn);
    if ((long long)p->N * make_plan(*p).w_pieces >= (1ll << 24)) return fail(FDD_ERR_SHAPE, "%s: N*V too large", kFn);
    if (p->dtype != FDD_F32 && p->dtype != FDD_BF16) return fail(FDD_ERR_DTYPE, "%s: dtype %d is neither FDD_F32 nor FDD_BF16", kFn, p->dtype);
    if (p->reserved != 0) return fail(FDD_ERR_UNSUPPORTED, "%s: reserved field must be 0", kFn);
    if (p->temperature != 0.f && !in_range(p->temperature)) return fail(FDD_ERR_UNSUPPORTED, "%s: temperature must be 0 (greedy) or from 2^-20 to 2^20", kFn);
    if (p->draft_logits && p->temperature != 0.f && !in_range(p->draft_temperature)) return fail(FDD_ERR_UNSUPPORTED, "%s: draft_temperature must be from 2^-20 to 2^20", kFn);
    return FDD_OK;
}

}  // namespace

extern "C" {

size_t fdd_tree_verify_workspace(const fdd_tree_verify_params* p)
{
    if (check_shape(p) != FDD_OK) return 0;
    const Plan pl = make_plan(*p);
    return pl.stats + pl.stops + pl.lists + pl.sums;
}

fdd_status fdd_tree_verify(const fdd_tree_verify_params* p)
{
    const fdd_status st = check_shape(p);
    if (st != FDD_OK) return st;
    const bool greedy = p->temperature == 0.f;
    if (!p->logits || !p->tokens || !p->path || !p->n_path || !p->emitted || (!greedy && !p->uniforms))
        return fail(FDD_ERR_NULL, "%s: logits, tokens, path, n_path and emitted must not be NULL, nor uniforms where the temperature is not 0", kFn);
    if (!greedy && p->draft_logits && p->parents) return fail(FDD_ERR_UNSUPPORTED, "%s: draft_logits go with chains only (parents must be NULL)", kFn);
    if (p->parents && p->parents_stride != 0 && (p->parents_stride < p->B || p->parents_stride > (1ll << 28)))
        return fail(FDD_ERR_SHAPE, "%s: parents_stride=%lld must be 0, or at least B=%d and at most 2^28", kFn, (long long)p->parents_stride, p->B);
    const uintptr_t es = (uintptr_t)dtype_bytes(p->dtype);
    if (!aligned_to(p->logits, es) || !aligned_to(p->draft_logits, es)) return fail(FDD_ERR_UNSUPPORTED, "%s: logits must be aligned to their element type", kFn);
    const void* lists[] = {p->tokens, p->parents, p->uniforms, p->n_tokens, p->path, p->n_path, p->emitted, p->chances};
    for (const void* x : lists)
        if (!aligned_to(x, 4)) return fail(FDD_ERR_UNSUPPORTED, "%s: arrays must be 4-byte aligned", kFn);
    const Plan pl = make_plan(*p);
    const size_t need = pl.stats + pl.stops + pl.lists + pl.sums;
    if (!p->workspace) return fail(FDD_ERR_WORKSPACE, "%s: workspace is NULL, %zu bytes needed", kFn, need);
    if (!aligned_to(p->workspace, 256)) return fail(FDD_ERR_WORKSPACE, "%s: workspace must be 256-byte aligned", kFn);
    if (p->workspace_bytes < need) return fail(FDD_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", kFn, p->workspace_bytes, need);
    const unsigned long long N = p->N, B = p->B, rows = N * B * 4, logits = N * B * (unsigned long long)p->V * es;
    const Span outs[] = {{p->path, rows}, {p->n_path, N * 4}, {p->emitted, rows}, {p->chances, rows}, {p->workspace, need}};
    const Span ins[] = {{p->logits, logits}, {greedy ? nullptr : p->draft_logits, logits}, {p->tokens, rows}, {p->parents, ((N - 1) * p->parents_stride + B) * 4},
                        {greedy ? nullptr : p->uniforms, 2 * rows}, {p->n_tokens, N * 4}};
    if (outputs_overlap(outs, ins)) return fail(FDD_ERR_UNSUPPORTED, "%s: an output or the workspace overlaps another array", kFn);
    Args a = {};
    a.logits = p->logits; a.draft = greedy ? nullptr : p->draft_logits; a.tokens = p->tokens; a.parents = p->parents; a.parents_stride = p->parents_stride;
    a.uniforms = p->uniforms; a.n_tokens = p->n_tokens; a.path = p->path; a.n_path = p->n_path; a.emitted = p->emitted; a.chances = p->chances;
    char* const ws = static_cast<char*>(p->workspace);
    a.stats = reinterpret_cast<Stat*>(ws);
    a.stops = reinterpret_cast<Stop*>(ws + pl.stats);
    a.lists = reinterpret_cast<int32_t*>(ws + pl.stats + pl.stops);
    a.sums = reinterpret_cast<double*>(ws + pl.stats + pl.stops + pl.lists);
    a.N = p->N; a.B = p->B; a.V = (int)p->V; a.pieces = pl.pieces; a.per_piece = pl.per_piece;
    a.w_pieces = pl.w_pieces; a.w_per = pl.w_per;
    if (!greedy) {
        a.c64 = LOG2E / (double)p->temperature;
        a.c = (float)a.c64;
        a.slack = 8.f / a.c;
    }
    if (a.draft) {
        a.draft_c64 = LOG2E / (double)p->draft_temperature;
        a.draft_c = (float)a.draft_c64;
        a.draft_slack = 8.f / a.draft_c;
    }
    const hipStream_t s = static_cast<hipStream_t>(p->stream);
    const hipError_t e = p->dtype == FDD_BF16 ? launch<uint16_t>(a, greedy, s) : launch<float>(a, greedy, s);
    if (e != hipSuccess) return fail(FDD_ERR_LAUNCH, "%s: launch failed: %s", kFn, hipGetErrorString(e));
    return FDD_OK;
}

}  // extern "C"
