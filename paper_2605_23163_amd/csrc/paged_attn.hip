// Attention of every request's new tokens over its paged cache and over one another (fdd_paged_attn), gfx950 matrix cores.
//
// How the work is laid out
//   * The query rows of a request and a KV head, r = token * G + g, are cut into M-tiles of WAVES * 32 rows, 32 for each
//     wavefront.  All of them use every tile of keys that the workgroup brings into LDS.
//   * Keys come in tiles: those of the cache, then those of the request's own tokens.  How many a request has is known on the
//     device only (lens, n_tokens): each workgroup works out for itself, from these two lists, how many tiles there are in
//     all, how many of them a piece gets so that all pieces together are as many as the chip takes at once, and which
//     piece is its own (`Cutting`).  A long request is cut into more pieces than a short one; the host only knows a bound.
//   * Scores are produced transposed, S^T = K Q^T, with 32x32 matrix instructions: each lane then owns one query row
//     (lane % 32) and half of the keys, so that maximum and sum of the streaming softmax are in-lane reductions plus
//     one exchange between the halves, and the same registers are the B operand of O^T += V^T P^T.
//   * A tile goes from global memory straight into LDS, in pieces of 1 KB for each wavefront instruction.  A piece lies in one page (4
//     or more rows of 16 and more); the page's number is uniform and stands in the descriptor's 64-bit base, so that the pool may
//     have any size.  Rows behind the last one repeat it: what lies behind it in the page is not read.
//   * bf16: 32x32x16 instructions, tiles of 64 keys.  K's 16-byte pieces are XOR-swizzled by the row, V's 32-byte columns too, which V's
//     transposing LDS reads (ds_read_b64_tr_b16) need.  fp32: 32x32x2 instructions, tiles of 32 keys; V is read as it lies.
//   * The softmax reference of a row rises only when a score passes it by more than 2^8: the accumulator is rarely rescaled.
//   * A request whose tiles are one piece is normalised and written at once; otherwise pieces leave fp32 sums and (m, l), which
//     merge_kernel joins in the order of the pieces.
#include <type_traits>

#include "paged.h"
#include "wave.h"

namespace fdd {
namespace paged_attn {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

constexpr uint32_t RSRC_FLAGS = 0x00020000;
constexpr int MIN_TILES = 2;        // a piece has no fewer, as long as there are more

// What decides how the work is cut: the same for the attention and the merge kernel.
struct Cut {
    const int32_t* lens;
    const int32_t* n_tokens;
    int N, B, G, Hkv;
    int max_len;        // longer requests are cut here
    int W;              // pieces aimed at
};

struct Args {
    Cut cut;
    const void* q;
    const void* bk;
    const void* bv;
    const void* k_pages;
    const void* v_pages;
    const int32_t* table;
    const uint64_t* mask;
    void* out;
    float* ws_o;        // [item][wave][D / 4 / 2 pieces][lane] of 16 bytes: accumulators as they stand
    float* ws_ml;       // [item][row][2]
    long long q_stride, k_stride, v_stride, mask_stride;
    int pages, page_shift, max_pages, Hq;
    int causal;
    float c;            // scale * log2(e)
    float slack;        // 8 / c
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float other_half(float x)
{
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_bit_cast(float, (thread_id_x() & 32) ? r[0] : r[1]);
}
template <int N>
__device__ __forceinline__ void wait_loads()      // until at most N of this wavefront's are on their way
{
    static_assert(N >= 0 && N < 64, "counter range");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | ((N >> 4) << 14));
}
__device__ __forceinline__ void wg_barrier() { asm volatile("s_barrier" ::: "memory"); }
__device__ __forceinline__ i16x4 read_tr(const lds_i16x4* __restrict__ p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(const_cast<lds_i16x4*>(p));
}

struct Request {
    int len, count;     // rows of the cache, new tokens
    int mtiles, tiles;  // M-tiles of a KV head; tiles of keys
};
template <typename C>
__device__ __forceinline__ Request request(const Cut& c, int n)
{
    Request r;
    r.len = min(max(c.lens[n], 0), c.max_len);
    r.count = c.n_tokens ? min(max(c.n_tokens[n], 0), c.B) : c.B;
    r.mtiles = (r.count * c.G + C::MROWS - 1) / C::MROWS;
    r.tiles = (r.len + C::KT - 1) / C::KT + (r.count + C::KT - 1) / C::KT;
    return r;
}

__device__ __forceinline__ int wave_sum(int x) { return (int)wave_reduce((uint32_t)x, [](uint32_t p, uint32_t q) { return p + q; }); }
__device__ __forceinline__ int wave_scan(int x, int lane)      // inclusive
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

struct Piece {
    int n, kh, mt, piece, pieces;      // n < 0: none
    int item;                          // its place among all
    Request r;
};

// How all requests are cut.  Lane n holds request n of the first 64; others are read again where they are needed.
template <typename C>
struct Cutting {
    Request r;
    int per_piece;      // tiles of a piece, at most

    __device__ __forceinline__ int pieces_of(const Request& x) const { return (x.tiles + per_piece - 1) / per_piece; }
    __device__ __forceinline__ int items_of(const Cut& c, const Request& x) const { return c.Hkv * x.mtiles * pieces_of(x); }
    // Tiles of a piece: all tiles over the pieces aimed at.
    __device__ __forceinline__ void set(const Cut& c, int lane)
    {
        r = {0, 0, 0, 0};
        if (lane < c.N) r = request<C>(c, lane);
        int tiles = r.mtiles * r.tiles;
        for (int n = 64 + lane; n < c.N; n += 64) {
            const Request x = request<C>(c, n);
            tiles += x.mtiles * x.tiles;
        }
        const int all = wave_sum(tiles) * c.Hkv;
        per_piece = max(MIN_TILES, __builtin_amdgcn_readfirstlane((all + c.W - 1) / c.W));
    }
    // The item-th piece.  Items of a request are ordered by (KV head, piece, M-tile).  Workgroups take them as they come, neighbours
    // on different XCDs: with neighbours on one XCD, whose M-tiles then share keys in its L2, 16 requests of one token and up to
    // 8192 rows took 54 us instead of 45, and 16 of 64 tokens and 16384 rows 310 instead of 301.
    __device__ __forceinline__ Piece find(const Cut& c, int lane, int item) const
    {
        const int items0 = items_of(c, r), end0 = wave_scan(items0, lane);
        Piece p;
        p.n = -1;
        p.item = item;
        Request x = r;
        int items = items0, end = end0;
        for (int n0 = 0;;) {
            const uint64_t here = __builtin_amdgcn_ballot_w64(item >= end - items && item < end);
            if (here) {
                const int l = __builtin_ctzll(here);
                auto of = [&](int y) { return __builtin_amdgcn_readlane(y, l); };
                p.n = n0 + l;
                p.r = {of(x.len), of(x.count), of(x.mtiles), of(x.tiles)};
                p.pieces = of(pieces_of(x));
                const int in = item - of(end - items);
                const int rest = in / p.r.mtiles;
                p.mt = in - rest * p.r.mtiles;
                p.kh = rest / p.pieces;
                p.piece = rest - p.kh * p.pieces;
                return p;
            }
            n0 += 64;
            if (n0 >= c.N) return p;
            const int base = __builtin_amdgcn_readlane(end, 63);
            x = {0, 0, 0, 0};
            if (n0 + lane < c.N) x = request<C>(c, n0 + lane);
            items = items_of(c, x);
            end = base + wave_scan(items, lane);
        }
    }
};

template <typename T, int D, int WAVES>
struct Cfg {
    static constexpr bool BF16 = std::is_same<T, uint16_t>::value;
    static constexpr int KT = BF16 ? 64 : 32;            // keys per tile
    static constexpr int MROWS = WAVES * 32;             // rows per M-tile
    static constexpr int ROW = D * (int)sizeof(T);       // bytes
    static constexpr int T_BYTES = KT * ROW;             // 16 KB at D = 128
    static constexpr int CH = ROW / 16;                  // 16-byte pieces per row
    static constexpr int RPB = 1024 / ROW;               // rows per 1 KB piece
    static constexpr int RPL = ROW < 256 ? 256 / ROW : 1;      // rows per 256-byte bank line
    static constexpr int NI = T_BYTES / 1024 / WAVES;    // pieces per wavefront, tile and operand
    static constexpr int SLOTS = WAVES == 8 ? 3 : 2;
    static constexpr int V_RING = SLOTS * T_BYTES;
    static constexpr int LDS = 2 * SLOTS * T_BYTES;
    static_assert(NI >= 1, "a tile has a piece for every wavefront");
};

template <typename T, int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void attn_kernel(Args a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using C = Cfg<T, D, WAVES>;
    constexpr int KT = C::KT, DB = D / 32;
    extern __shared__ __align__(16) unsigned char lds[];
    const int tid = thread_id_x(), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // ---- this workgroup's piece --------------------------------------------------------------------------------------
    Cutting<C> cutting;
    cutting.set(a.cut, lane);
    const Piece p = cutting.find(a.cut, lane, (int)wg_id_x());
    if (p.n < 0) return;
    const int n = p.n, kh = p.kh, len = p.r.len, count = p.r.count;
    const int cache_tiles = (len + KT - 1) / KT;
    int t_begin = (int)((long long)p.r.tiles * p.piece / p.pieces), t_end = (int)((long long)p.r.tiles * (p.piece + 1) / p.pieces);
    t_begin = __builtin_amdgcn_readfirstlane(t_begin);
    t_end = __builtin_amdgcn_readfirstlane(t_end);

    // ---- rows ----------------------------------------------------------------------------------------------------------
    const int G = a.cut.G, rows = count * G;
    const int row0 = p.mt * (WAVES * 32);
    const int row = row0 + wave * 32 + l32;
    const bool row_ok = row < rows;
    const int row_c = min(row, rows - 1);
    const int token = row_c / G, g = row_c - token * G;
    if (a.causal) {      // keys behind the M-tile's last token are not seen
        const int last = (min(row0 + WAVES * 32, rows) - 1) / G;
        t_end = min(t_end, cache_tiles + last / KT + 1);
    }
    const int W64 = (a.cut.B + 63) >> 6;
    const uint64_t* const bits = a.mask ? a.mask + n * a.mask_stride + (long long)token * W64 : nullptr;

    // ---- tiles: global memory -> LDS --------------------------------------------------------------------------------------
    // page numbers of the next 64 pages, one a lane
    const int32_t* const table = a.table + (long long)n * a.max_pages;
    int window = -1, entries = 0;
    auto page_at = [&](int index) -> int {
        if ((index >> 6) != window) {
            window = index >> 6;
            entries = table[min((window << 6) + lane, a.max_pages - 1)];
            entries = min(max(entries, 0), a.pages - 1);
        }
        return __builtin_amdgcn_readlane(entries, index & 63);
    };
    const uint32_t page_bytes = (uint32_t)C::ROW << a.page_shift;
    const int page_mask = (1 << a.page_shift) - 1;
    // chunk of row r that lands at 16-byte piece `at` of its place in LDS
    auto k_chunk = [&](int at, int r) { return at ^ ((r / C::RPL) & (C::CH - 1)); };
    auto v_chunk = [&](int at, int r) { return C::BF16 ? at ^ ((((r / C::RPL) & 3) << 2) & (C::CH - 1)) : at; };
    const int lane_row = lane / C::CH, lane_at = lane % C::CH;
    auto fetch = [&](int t, int slot) {
        unsigned char* const dst = lds + slot * C::T_BYTES + wave * (C::NI * 1024);
        if (t < cache_tiles) {
#pragma unroll
            for (int i = 0; i < C::NI; ++i) {
                const int r0 = (wave * C::NI + i) * C::RPB, r = r0 + lane_row;
                const int first = min(t * KT + r0, len - 1);      // (a piece behind the last row repeats it)
                const int page = page_at(first >> a.page_shift);
                const long long at = ((long long)page * a.cut.Hkv + kh) * page_bytes;
                const uint32_t in_page = (uint32_t)(min(t * KT + r, len - 1) & page_mask) * C::ROW;
                const __amdgpu_buffer_rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(a.k_pages)) + at, 0, page_bytes, RSRC_FLAGS);
                const __amdgpu_buffer_rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(a.v_pages)) + at, 0, page_bytes, RSRC_FLAGS);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (lds_void*)(dst + i * 1024), 16, in_page + k_chunk(lane_at, r) * 16, 0, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (lds_void*)(dst + C::V_RING + i * 1024), 16, in_page + v_chunk(lane_at, r) * 16, 0, 0, 0);
            }
        } else {
            const int key0 = (t - cache_tiles) * KT, last = count - 1 - key0;
            const char* const kb = static_cast<const char*>(a.bk) + (((long long)n * a.cut.B + key0) * a.k_stride + kh * D) * (long long)sizeof(T);
            const char* const vb = static_cast<const char*>(a.bv) + (((long long)n * a.cut.B + key0) * a.v_stride + kh * D) * (long long)sizeof(T);
            const __amdgpu_buffer_rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(kb), 0, 0xffffffffu, RSRC_FLAGS);
            const __amdgpu_buffer_rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(vb), 0, 0xffffffffu, RSRC_FLAGS);
#pragma unroll
            for (int i = 0; i < C::NI; ++i) {
                const int r = (wave * C::NI + i) * C::RPB + lane_row;
                const uint32_t rr = (uint32_t)min(r, last);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (lds_void*)(dst + i * 1024), 16, rr * (uint32_t)a.k_stride * (uint32_t)sizeof(T) + k_chunk(lane_at, r) * 16, 0, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (lds_void*)(dst + C::V_RING + i * 1024), 16, rr * (uint32_t)a.v_stride * (uint32_t)sizeof(T) + v_chunk(lane_at, r) * 16, 0, 0, 0);
            }
        }
    };

    // ---- queries: B operand of S^T = K Q^T --------------------------------------------------------------------------------
    constexpr int QF = D * (int)sizeof(T) / 32;       // 16-byte fragments of a lane: half of a row
    u32x4 qf[QF];
    {
        const char* const qp = static_cast<const char*>(a.q) + (((long long)n * a.cut.B + token) * a.q_stride + (kh * G + g) * D) * (long long)sizeof(T) + half * 16;
#pragma unroll
        for (int i = 0; i < QF; ++i) qf[i] = *reinterpret_cast<const u32x4*>(qp + i * 32);
    }

    // ---- streaming softmax: one query row per lane ---------------------------------------------------------------------------
    f32x16 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[db][v] = 0.f;
    float m_ref = 0.f, limit = -INFINITY, l_run = 0.f;
    auto update_reference = [&](float mx) {
        if (__any(mx > limit)) {
            const bool none = limit == -INFINITY;
            float m = fmaxf(mx, other_half(mx));
            if (!none) m = fmaxf(m, m_ref);
            const float alpha = none ? 0.f : exp2_fast((m_ref - m) * a.c);
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[db][v] *= alpha;
            m_ref = m == -INFINITY ? 0.f : m;
            limit = m == -INFINITY ? m : m + a.slack;
        }
    };

    const int k_off = l32 * C::ROW, k_swz = (l32 / C::RPL) & (C::CH - 1);
    int v_off[DB];
    {
        const int row_l = half * 4 + ((lane & 15) >> 2), x = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
        const int sw = (((row_l / C::RPL) & 3) << 2) & (C::CH - 1);
#pragma unroll
        for (int db = 0; db < DB; ++db) v_off[db] = (row_l * C::ROW + ((x ^ sw) << 4) + (lane & 1) * 8) ^ (db << 6);
    }

    constexpr int KB = KT / 32;
    auto step = [&](int t, int slot) {
        const unsigned char* const kt = lds + slot * C::T_BYTES;
        const unsigned char* const vt = kt + C::V_RING;
        f32x16 s[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
            for (int v = 0; v < 16; ++v) s[kb][v] = 0.f;
#pragma unroll
            for (int i = 0; i < QF; ++i) {
                const u32x4 kf = *reinterpret_cast<const u32x4*>(kt + kb * 32 * C::ROW + k_off + (((2 * i + half) ^ k_swz) << 4));
                if constexpr (C::BF16) {
                    s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[i]), s[kb], 0, 0, 0);
                } else {
                    const f32x4 kx = __builtin_bit_cast(f32x4, kf), qx = __builtin_bit_cast(f32x4, qf[i]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(kx[j], qx[j], s[kb], 0, 0, 0);
                }
            }
        }
        // keys that the row does not see
        const bool cache = t < cache_tiles;
        const int key0 = cache ? t * KT : (t - cache_tiles) * KT;
        const int valid = cache ? len - key0 : count - key0;
        if (!cache || valid < KT) {
            uint64_t see = valid >= 64 ? ~0ull : (1ull << valid) - 1;
            if (!cache) {
                if (bits) see &= bits[key0 >> 6] >> (key0 & 63);
                else if (a.causal) see &= token - key0 >= 63 ? ~0ull : token < key0 ? 0ull : (2ull << (token - key0)) - 1;
            }
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {
                const uint32_t w = (uint32_t)(see >> (32 * kb + 4 * half));
#pragma unroll
                for (int v = 0; v < 16; ++v) s[kb][v] = (w >> (8 * (v / 4) + v % 4)) & 1 ? s[kb][v] : -INFINITY;
            }
        }
        float mx = s[0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[kb][v]);
        update_reference(mx);
        const float mc = m_ref * a.c;
        float sum = 0.f;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                s[kb][v] = exp2_fast(fmaf(s[kb][v], a.c, -mc));
                sum += s[kb][v];
            }
        l_run += sum;
        if constexpr (C::BF16) {
#pragma unroll
            for (int t4 = 0; t4 < KT / 16; ++t4) {
                bf16x8 pf;
#pragma unroll
                for (int e = 0; e < 8; ++e) pf[e] = (__bf16)s[t4 / 2][(t4 & 1) * 8 + e];
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const unsigned char* const vp = vt + v_off[db] + t4 * 16 * C::ROW;
                    const i16x4 lo = read_tr((const lds_i16x4*)vp), hi = read_tr((const lds_i16x4*)(vp + 8 * C::ROW));
                    typedef short i16x8 __attribute__((ext_vector_type(8)));
                    const i16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, both), pf, o[db], 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const unsigned char* const vp = vt + (8 * (v / 4) + 4 * half + v % 4) * C::ROW + l32 * 4;
#pragma unroll
                for (int db = 0; db < DB; ++db)
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float*>(vp + db * 128), s[0][v], o[db], 0, 0, 0);
            }
        }
    };

    // ---- the piece's tiles -----------------------------------------------------------------------------------------------
    constexpr int LOADS = 2 * C::NI;
#pragma unroll
    for (int i = 0; i < C::SLOTS - 1; ++i)
        if (t_begin + i < t_end) fetch(t_begin + i, i);
    // (the queries are here from now on: otherwise each step's first use of them waits for the tiles on their way too)
#pragma unroll
    for (int i = 0; i < QF; ++i) asm volatile("" : "+v"(qf[i]));
    int slot = 0;
    for (int t = t_begin; t < t_end; ++t) {
        if (C::SLOTS == 3 && t + 1 < t_end) wait_loads<LOADS>();
        else wait_loads<0>();
        wg_barrier();       // the tile is there, and everyone is done with the slot that the next one goes to
        if (t + C::SLOTS - 1 < t_end) fetch(t + C::SLOTS - 1, slot == 0 ? C::SLOTS - 1 : slot - 1);
        step(t, slot);
        slot = slot + 1 == C::SLOTS ? 0 : slot + 1;
    }

    // ---- out ---------------------------------------------------------------------------------------------------------------
    const float l = l_run + other_half(l_run);
    if (p.pieces == 1) {
        if (!row_ok) return;
        const float inv = l > 0.f ? 1.f / l : 0.f;
        T* const op = static_cast<T*>(a.out) + (((long long)n * a.cut.B + token) * a.Hq + kh * G + g) * D + 4 * half;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int v4 = 0; v4 < 4; ++v4) {
                float x[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = l > 0.f ? o[db][4 * v4 + j] * inv : 0.f;
                if constexpr (C::BF16) {
                    u32x2 w;
                    w[0] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[0]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[1]) << 16;
                    w[1] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[2]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[3]) << 16;
                    *reinterpret_cast<u32x2*>(op + db * 32 + v4 * 8) = w;
                } else {
                    *reinterpret_cast<f32x4*>(op + db * 32 + v4 * 8) = f32x4{x[0], x[1], x[2], x[3]};
                }
            }
    } else if (row_ok) {
        f32x4* const wo = reinterpret_cast<f32x4*>(a.ws_o) + ((long long)p.item * WAVES + wave) * (DB * 4 * 64) + lane;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int v4 = 0; v4 < 4; ++v4) wo[(db * 4 + v4) * 64] = f32x4{o[db][4 * v4], o[db][4 * v4 + 1], o[db][4 * v4 + 2], o[db][4 * v4 + 3]};
        if (half == 0) {
            float* const ml = a.ws_ml + ((long long)p.item * WAVES * 32 + wave * 32 + l32) * 2;
            ml[0] = l > 0.f ? m_ref * a.c : -INFINITY;
            ml[1] = l;
        }
    }
#endif
}

struct MergeArgs {
    Cut cut;
    const float* ws_o;
    const float* ws_ml;
    void* out;
    int Hq, max_mt;
};

// One wavefront per (request, KV head, M-tile, its 32-row wavefront, MERGE_COLS of its 16-byte columns): lane = as in the accumulators.
// Bound by latency where pieces are many: UNROLL of them are on their way at a time.
constexpr int MERGE_COLS = 2, UNROLL = 8;
template <typename T, int D, int WAVES>
__global__ __launch_bounds__(256) void merge_kernel(MergeArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using C = Cfg<T, D, WAVES>;
    constexpr int COLS = D / 8, GROUPS = COLS / MERGE_COLS;
    const int tid = thread_id_x(), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
    int job = __builtin_amdgcn_readfirstlane((int)wg_id_x() * 4 + (tid >> 6));
    const int col0 = job % GROUPS * MERGE_COLS;
    job /= GROUPS;
    const int wave = job % WAVES, mtile = job / WAVES;
    const int mt = mtile % a.max_mt, head = mtile / a.max_mt;
    const int n = head / a.cut.Hkv, kh = head - n * a.cut.Hkv;
    if (n >= a.cut.N) return;
    Cutting<C> cutting;
    cutting.set(a.cut, lane);
    int before = lane < n ? cutting.items_of(a.cut, cutting.r) : 0;
    Request x = cutting.r;
    for (int n0 = 64; n0 <= n; n0 += 64) {
        x = {0, 0, 0, 0};
        if (n0 + lane <= n) x = request<C>(a.cut, n0 + lane);
        if (n0 + lane < n) before += cutting.items_of(a.cut, x);
    }
    const int base = wave_sum(before), l = n & 63;
    const Request mine = {__builtin_amdgcn_readlane(x.len, l), __builtin_amdgcn_readlane(x.count, l), __builtin_amdgcn_readlane(x.mtiles, l),
                          __builtin_amdgcn_readlane(x.tiles, l)};
    const int pieces = cutting.pieces_of(mine);
    if (pieces <= 1 || mt >= mine.mtiles) return;
    const int row = (mt * WAVES + wave) * 32 + l32;
    const bool row_ok = row < mine.count * a.cut.G;
    if (!row_ok) return;
    const int first = base + (kh * pieces) * mine.mtiles + mt;
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2* const ml0 = reinterpret_cast<const f32x2*>(a.ws_ml) + ((long long)first * WAVES + wave) * 32 + l32;
    const f32x4* const wo0 = reinterpret_cast<const f32x4*>(a.ws_o) + (((long long)first * WAVES + wave) * COLS + col0) * 64 + lane;
    const long long ml_step = (long long)mine.mtiles * WAVES * 32, wo_step = (long long)mine.mtiles * WAVES * COLS * 64;
    float m = -INFINITY, l_sum = 0.f;
    f32x4 y[MERGE_COLS];
#pragma unroll
    for (int j = 0; j < MERGE_COLS; ++j) y[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < pieces; i += UNROLL) {
        f32x2 ml[UNROLL];
        f32x4 w[UNROLL][MERGE_COLS];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int at = min(i + u, pieces - 1);
            ml[u] = ml0[at * ml_step];
#pragma unroll
            for (int j = 0; j < MERGE_COLS; ++j) w[u][j] = wo0[at * wo_step + j * 64];
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (i + u >= pieces) ml[u][0] = -INFINITY;
            top = fmaxf(top, ml[u][0]);
        }
        const float ref = top == -INFINITY ? 0.f : top;
        const float old = exp2_fast(m - ref);
        m = top;
        l_sum *= old;
#pragma unroll
        for (int j = 0; j < MERGE_COLS; ++j) y[j] = f32x4{y[j][0] * old, y[j][1] * old, y[j][2] * old, y[j][3] * old};
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const float f = exp2_fast(ml[u][0] - ref);
            l_sum = fmaf(f, ml[u][1], l_sum);
#pragma unroll
            for (int j = 0; j < MERGE_COLS; ++j) {
                const f32x4 z = w[u][j];
                y[j] = f32x4{fmaf(f, z[0], y[j][0]), fmaf(f, z[1], y[j][1]), fmaf(f, z[2], y[j][2]), fmaf(f, z[3], y[j][3])};
            }
        }
    }
    const int token = row / a.cut.G, g = row - token * a.cut.G;
    const float inv = l_sum > 0.f ? 1.f / l_sum : 0.f;
    T* const op = static_cast<T*>(a.out) + (((long long)n * a.cut.B + token) * a.Hq + kh * a.cut.G + g) * D + 4 * half + col0 * 8;
#pragma unroll
    for (int j = 0; j < MERGE_COLS; ++j) {
        float z[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = l_sum > 0.f ? y[j][e] * inv : 0.f;
        if constexpr (std::is_same<T, float>::value) {
            *reinterpret_cast<f32x4*>(op + j * 8) = f32x4{z[0], z[1], z[2], z[3]};
        } else {
            u32x2 w;
            w[0] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)z[0]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)z[1]) << 16;
            w[1] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)z[2]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)z[3]) << 16;
            *reinterpret_cast<u32x2*>(op + j * 8) = w;
        }
    }
#endif
}

// ---- host ----------------------------------------------------------------------------------------------------------------

struct Plan {
    int waves, kt, max_mt, W;
    int max_len;
    long long items;            // no call has more pieces
    bool partials;              // some request may have more than one piece
    size_t o_bytes, ml_bytes;
};

Plan make_plan(const fdd_paged_cache& c, const fdd_paged_attn_params& p)
{
    Plan pl;
    const long long rows = (long long)p.B * (p.Hq / c.Hkv);
    pl.waves = rows <= 32 ? 1 : rows <= 64 ? 2 : rows <= 128 ? 4 : 8;
    pl.kt = c.dtype == FDD_BF16 ? 64 : 32;
    const int capacity = c.max_pages * c.page_size;
    pl.max_len = p.max_len > 0 ? (p.max_len < capacity ? p.max_len : capacity) : capacity;
    pl.max_mt = (int)((rows + pl.waves * 32 - 1) / (pl.waves * 32));
    pl.W = pl.waves == 8 ? kNumCU : 2 * kNumCU;
    const long long tiles = (pl.max_len + pl.kt - 1) / pl.kt + (p.B + pl.kt - 1) / pl.kt;
    const long long mtiles = (long long)c.N * c.Hkv * pl.max_mt;
    pl.partials = tiles > MIN_TILES;
    pl.items = mtiles + (pl.partials ? pl.W : 0);
    const size_t prow = pl.partials ? (size_t)pl.items * pl.waves * 32 : 0;
    pl.o_bytes = (prow * c.D * 4 + 255) & ~(size_t)255;
    pl.ml_bytes = (prow * 8 + 255) & ~(size_t)255;
    return pl;
}

Cut make_cut(const fdd_paged_cache& c, const fdd_paged_attn_params& p, const Plan& pl)
{
    return {c.lens, p.n_tokens, c.N, p.B, p.Hq / c.Hkv, c.Hkv, pl.max_len, pl.W};
}

template <typename T, int D, int WAVES>
hipError_t launch(const fdd_paged_cache& c, const fdd_paged_attn_params& p, const Plan& pl, const Args& a)
{
    using C = Cfg<T, D, WAVES>;
    const hipStream_t s = static_cast<hipStream_t>(p.stream);
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(attn_kernel<T, D, WAVES>), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
    if (e != hipSuccess) return e;
    attn_kernel<T, D, WAVES><<<dim3((unsigned)pl.items), WAVES * 64, C::LDS, s>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess || !pl.partials) return e;
    MergeArgs m = {a.cut, a.ws_o, a.ws_ml, p.out, p.Hq, pl.max_mt};
    const long long jobs = (long long)c.N * c.Hkv * pl.max_mt * WAVES * (D / 8 / MERGE_COLS);
    merge_kernel<T, D, WAVES><<<dim3((unsigned)((jobs + 3) / 4)), 256, 0, s>>>(m);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_waves(const fdd_paged_cache& c, const fdd_paged_attn_params& p, const Plan& pl, const Args& a)
{
    switch (pl.waves) {
    case 1: return launch<T, D, 1>(c, p, pl, a);
    case 2: return launch<T, D, 2>(c, p, pl, a);
    case 4: return launch<T, D, 4>(c, p, pl, a);
    default: return launch<T, D, 8>(c, p, pl, a);
    }
}

}  // namespace paged_attn
}  // namespace fdd

using namespace fdd;
using namespace fdd::paged_attn;

#define fail set_error

namespace {

const char* const kFn = "fdd_paged_attn";

fdd_status check_shape(const fdd_paged_cache* c, const fdd_paged_attn_params* p)
{
    const fdd_status st = check_paged_cache(c, kFn);
    if (st != FDD_OK) return st;
    if (!p) return fail(FDD_ERR_NULL, "%s: params is NULL", kFn);
    if (p->B <= 0 || p->Hq <= 0 || p->max_len < 0) return fail(FDD_ERR_SHAPE, "%s: B and Hq must be positive and max_len >= 0 (got B=%d Hq=%d max_len=%d)", kFn, p->B, p->Hq, p->max_len);
    if (p->Hq % c->Hkv) return fail(FDD_ERR_SHAPE, "%s: Hq=%d is not a multiple of Hkv=%d", kFn, p->Hq, c->Hkv);
    if (p->flags & ~FDD_ATTN_CAUSAL_BLOCK) return fail(FDD_ERR_UNSUPPORTED, "%s: unknown bits in flags (0x%x)", kFn, p->flags);
    if (p->reserved != 0) return fail(FDD_ERR_UNSUPPORTED, "%s: reserved field must be 0", kFn);
    if (!finite_bits(p->scale)) return fail(FDD_ERR_UNSUPPORTED, "%s: scale is not finite", kFn);
    const long long tokens = (long long)c->N * p->B;
    if (p->B > (1 << 24) || p->Hq > 65535 || tokens >= (1ll << 31) || tokens * p->Hq >= (1ll << 31)) return fail(FDD_ERR_SHAPE, "%s: N*B*Hq too large", kFn);
    const Plan pl = make_plan(*c, *p);
    const long long tiles = (pl.max_len + pl.kt - 1) / pl.kt + (p->B + pl.kt - 1) / pl.kt;
    if ((long long)c->N * c->Hkv * pl.max_mt * tiles >= (1ll << 31) - pl.W || pl.items >= (1ll << 22))
        return fail(FDD_ERR_SHAPE, "%s: N*B*Hq*max_len too large", kFn);
    return FDD_OK;
}

}  // namespace

extern "C" {

size_t fdd_paged_attn_workspace(const fdd_paged_cache* c, const fdd_paged_attn_params* p)
{
    if (check_shape(c, p) != FDD_OK) return 0;
    const Plan pl = make_plan(*c, *p);
    return pl.o_bytes + pl.ml_bytes;
}

fdd_status fdd_paged_attn(const fdd_paged_cache* c, const fdd_paged_attn_params* p)
{
    fdd_status st = check_shape(c, p);
    if (st != FDD_OK) return st;
    if (!p->q || !p->block_k || !p->block_v || !p->out) return fail(FDD_ERR_NULL, "%s: q, block_k, block_v and out must not be NULL", kFn);
    if (!aligned_to(p->q, 16) || !aligned_to(p->block_k, 16) || !aligned_to(p->block_v, 16) || !aligned_to(p->out, 16))
        return fail(FDD_ERR_UNSUPPORTED, "%s: data pointers must be 16-byte aligned", kFn);
    if (!aligned_to(p->mask, 8) || !aligned_to(p->n_tokens, 4)) return fail(FDD_ERR_UNSUPPORTED, "%s: mask must be 8-byte aligned, n_tokens 4-byte aligned", kFn);
    if (p->mask && (p->flags & FDD_ATTN_CAUSAL_BLOCK)) return fail(FDD_ERR_UNSUPPORTED, "%s: FDD_ATTN_CAUSAL_BLOCK does not go with a mask", kFn);
    const long long q_token = (long long)p->Hq * c->D, kv_token = (long long)c->Hkv * c->D, tokens = (long long)c->N * p->B, es = dtype_bytes(c->dtype);
    if ((st = check_token_stride(p->q_stride, q_token, c->dtype, "q_stride", kFn)) != FDD_OK) return st;
    if ((st = check_token_stride(p->k_stride, kv_token, c->dtype, "k_stride", kFn)) != FDD_OK) return st;
    if ((st = check_token_stride(p->v_stride, kv_token, c->dtype, "v_stride", kFn)) != FDD_OK) return st;
    // (a tile's tokens are reached by 32-bit offsets: 63 of these of 4 bytes)
    if (p->k_stride > (1 << 23) || p->v_stride > (1 << 23)) return fail(FDD_ERR_SHAPE, "%s: k_stride and v_stride must be at most 2^23 elements", kFn);
    const long long words = (long long)p->B * ((p->B + 63) / 64);
    if (p->mask && p->mask_stride != 0 && (p->mask_stride < words || p->mask_stride > (1ll << 40)))
        return fail(FDD_ERR_SHAPE, "%s: mask_stride=%lld must be 0 or at least %lld words", kFn, (long long)p->mask_stride, words);
    const Plan pl = make_plan(*c, *p);
    Args a = {};
    a.q_stride = token_stride(p->q_stride, q_token); a.k_stride = token_stride(p->k_stride, kv_token); a.v_stride = token_stride(p->v_stride, kv_token);
    const unsigned long long out_bytes = (unsigned long long)(tokens * q_token * es), pool = pool_bytes(*c);
    const struct { const void* p; unsigned long long bytes; } reads[] = {
        {p->q, (unsigned long long)(((tokens - 1) * a.q_stride + q_token) * es)}, {p->block_k, (unsigned long long)(((tokens - 1) * a.k_stride + kv_token) * es)},
        {p->block_v, (unsigned long long)(((tokens - 1) * a.v_stride + kv_token) * es)}, {c->k, pool}, {c->v, pool}};
    for (const auto& r : reads)
        if (spans_overlap(r.p, r.bytes, p->out, out_bytes)) return fail(FDD_ERR_UNSUPPORTED, "%s: out overlaps an input", kFn);
    const size_t need = pl.o_bytes + pl.ml_bytes;
    if (need > 0) {
        if (!p->workspace) return fail(FDD_ERR_WORKSPACE, "%s: workspace is NULL, %zu bytes needed", kFn, need);
        if (!aligned_to(p->workspace, 256)) return fail(FDD_ERR_WORKSPACE, "%s: workspace must be 256-byte aligned", kFn);
        if (p->workspace_bytes < need) return fail(FDD_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", kFn, p->workspace_bytes, need);
    }
    const float scale = p->scale > 0.f ? p->scale : 1.f / std::sqrt((float)c->D);
    a.cut = make_cut(*c, *p, pl);
    a.q = p->q; a.bk = p->block_k; a.bv = p->block_v; a.k_pages = c->k; a.v_pages = c->v; a.table = c->page_table; a.mask = p->mask; a.out = p->out;
    a.ws_o = static_cast<float*>(p->workspace);
    a.ws_ml = reinterpret_cast<float*>(static_cast<char*>(p->workspace) + pl.o_bytes);
    a.mask_stride = p->mask_stride;
    a.pages = c->pages; a.page_shift = __builtin_ctz((unsigned)c->page_size); a.max_pages = c->max_pages; a.Hq = p->Hq;
    a.causal = (p->flags & FDD_ATTN_CAUSAL_BLOCK) != 0;
    a.c = scale * 1.4426950408889634f;
    a.slack = 8.f / a.c;
    hipError_t e;
    if (c->dtype == FDD_BF16) e = c->D == 128 ? launch_waves<uint16_t, 128>(*c, *p, pl, a) : launch_waves<uint16_t, 64>(*c, *p, pl, a);
    else e = c->D == 128 ? launch_waves<float, 128>(*c, *p, pl, a) : launch_waves<float, 64>(*c, *p, pl, a);
    if (e != hipSuccess) return fail(FDD_ERR_LAUNCH, "%s: launch failed: %s", kFn, hipGetErrorString(e));
    return FDD_OK;
}

}  // extern "C"
