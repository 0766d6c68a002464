// Attention of every request's new tokens over its paged cache and over one another (fdd_paged_attn), gfx950 matrix cores.
//
// How the work is laid out
//   * The query rows of a request and a KV head, r = token * G + g, are cut into M-tiles of up to WAVES * 32 rows, as even as whole
//     wavefronts of 32 rows allow.  All of them use every tile of keys that the workgroup brings into LDS; wavefronts without rows only
//     help to bring it.
//   * Keys come in tiles: those of the cache, then those of the request's own tokens.  How many a request has is known on the
//     device only (lens, n_tokens): each workgroup works out for itself, from these two lists, how many tiles there are in
//     all, how many of them a piece gets, all over the W workgroups that the chip takes at once, and which
//     piece is its own (`Cutting`).  A long request is cut into more pieces than a short one; the host only knows a bound.  Both quotients are
//     rounded up, a piece's tiles and an M-tile's pieces, so that there are up to W + M-tiles pieces, and those beyond W wait for the others: with 64
//     tokens and 8192 rows 8 requests are 256 pieces of 33 tiles for W = 256, 74 us, 6 are 288 of 22, 86 us.
//   * Scores are produced transposed, S^T = K Q^T, with 32x32 matrix instructions: each lane then owns one query row
//     (lane % 32) and half of the keys, so that maximum and sum of the streaming softmax are in-lane reductions plus
//     one exchange between the halves, and the same registers are the B operand of O^T += V^T P^T.
//   * A tile goes from global memory straight into LDS, in pieces of 1 KB for each wavefront instruction.  A piece lies in one page (4
//     or more rows of 16 and more); the page's number is uniform and stands in the descriptor's 64-bit base, so that the pool may
//     have any size.  Rows behind the last one repeat it: what lies behind it in the page is not read.
//   * bf16: 32x32x16 instructions, tiles of 64 keys.  K's 16-byte pieces are XOR-swizzled by the row, V's 32-byte columns too, which V's
//     transposing LDS reads (ds_read_b64_tr_b16) need.  fp32: 32x32x2 instructions, tiles of 32 keys; V is read as it lies.
//   * The softmax reference of a row rises only when a score passes it by more than 2^8: the accumulator is rarely rescaled.
//   * A request whose tiles are one piece is normalised and written at once; otherwise pieces leave their sums and (m, l), which
//     merge_kernel joins in the order of the pieces.  bf16 calls leave averages in fp16 times a power of two for the row: off by 2^-11 of themselves or
//     2^-39 of the row's largest, where the output is rounded to 2^-8, in half the bytes, which can be as many as the keys'.  fp32 sums in their place
//     take 1 % or less off the error in norm (16 requests of one token 2.32e-3 -> 2.31e-3) and cost, us from a graph: 4 requests of 32 tokens and 4096 rows 23.3 -> 25.5,
//     16 of 8 and 8192 57.0 -> 60.8, 64 of one token and 1024 33.4 -> 34.9; 16 of one token and up to 8192 41.1 -> 40.7, one of 32768 22.6 -> 21.8.
//     fp32 calls leave sums.
//   * bf16 probabilities are rounded to bf16, which is what the matrix instructions take (summed as rounded): that and the output's rounding, 1.7e-3 in norm,
//     make 2.2e-3 to 2.4e-3 against 64 bits.
//
// Software pipeline (bf16): a step has the scores of tile t + 1 and, beside them in the same stretch of instructions, the softmax and O += P V of
// tile t; requests for later tiles stand between the matrix instructions.  A step of whole tiles has no branch.  Exponentials come in three
// stages spread over the slots, none waiting for the one before (16 requests of 64 tokens and 16384 rows 251 -> 245 us).
//
// Few rows have four wavefronts all the same, so that none makes a tile's 32 requests alone: 16 requests of one token and up to 8192 rows, the attention
// without the merge, 34.8 -> 29.6 us, 4 of 100 rows 12.1 -> 8.3.
//
// What bounds it (bf16, Hq / Hkv / D = 28 / 4 / 128).  Few rows: bytes, 5.6 TB/s in the attention, and the merge's launch: 16 requests of one token and
// up to 8192 rows 40.5 us, of them attention 29.7, merge 5.5 (floor 32.5 at the rate of a large copy).  Middle: a start of 5 us (lists, table, first
// requests): 4 x 32 tokens, 4096 rows 22.6 us (attention 16.2, merge 6.7).  Many rows: 16 x 64 tokens, 16384 rows 245 to 260 us, 985 to 928 TFLOP/s from card to card: the
// clock that the chip's power leaves, 1.7 to 1.85 GHz, and reads of LDS, without which the loop took 170 us of 237.  64 rows a wavefront, which
// read LDS half as often, leave one wavefront a SIMD: 339 us instead of 277 (as it was then).
// A prompt in one call: pieces are dealt as if every token saw all, and tiles of the request's own tokens take the steps with branches: 2048 tokens in order, no cache, 88 us
// (floor 25), each seeing all 95 (50), 2 x 512 behind 4096 rows 102 (53).
// fp32, matrix pipe: 3 x up to 21 tokens, 2003 rows, 14 / 2 / 64: 14.7 us (attention 10.5, merge 4.5).  16 x 1 token, 4096 rows, 28 / 4 / 128 83 us, floor
// 52: one wavefront of four has rows, and 7 of them.  A prompt of 1024 tokens in order 147 us, floor 49.
#pragma once
#include <atomic>
#include <type_traits>
#include <utility>

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
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

constexpr uint32_t RSRC_FLAGS = 0x00020000;
constexpr int MIN_TILES = 2;        // a piece has no fewer, as long as there are more

// What decides how the work is cut: the same for the attention and the merge kernel.
struct Cut {
    const int32_t* lens;
    const int32_t* n_tokens;
    int N, B, G, Hkv;
    FastDiv dG;
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
    float* ws_o;        // [item][wave][16-byte column][lane]: accumulators as they stand, fp32 sums or, of bf16 calls, fp16 averages
    float* ws_ml;       // [item][row][4]: reference, sum, factor of the averages
    long long q_stride, k_stride, v_stride, mask_stride;
    int used;           // wavefronts of an M-tile that can have rows: the others leave nothing
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
// The order of the source across this point is the order of the instructions.
#define SCHED_FENCE() __builtin_amdgcn_sched_barrier(0)
__device__ __forceinline__ void wg_barrier() { asm volatile("s_barrier" ::: "memory"); }
__device__ __forceinline__ i16x4 read_tr(const lds_i16x4* __restrict__ p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(const_cast<lds_i16x4*>(p));
}

// f(J0), f(J0 + 1), .. f(J1 - 1) with compile-time arguments
template <int J0, typename F, int... J>
__device__ __forceinline__ void each_of(const F& f, std::integer_sequence<int, J...>)
{
    (f(std::integral_constant<int, J0 + J>()), ...);
}
template <int J0, int J1, typename F>
__device__ __forceinline__ void each(const F& f)
{
    each_of<J0>(f, std::make_integer_sequence<int, J1 - J0>());
}

struct Request {
    int len, count;     // rows of the cache, new tokens
    int mtiles, tiles;  // M-tiles of a KV head; tiles of keys
};
// Rows of each of a request's M-tiles: as many, in whole wavefronts (448 rows are two M-tiles of 224, not of 256 and 192: wavefronts
// without rows leave the LDS and the matrix pipe to the others).
__device__ __forceinline__ int rows_per_mtile(int rows, int mtiles) { return ((rows + 31) / 32 + mtiles - 1) / mtiles * 32; }
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
__device__ __forceinline__ int wave_scan(int x)      // inclusive
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);      // row_shr 1, 2, 4, 8: rows of 16 lanes
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);     // row_bcast15: the last lane of rows 0 and 2 to rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);     // row_bcast31: lane 31 to rows 2 and 3
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
    // The item-th piece.  A request's (KV head, piece) pairs stand in groups of eight, and in a group one M-tile of all of them behind the
    // other: workgroups go to the XCDs in turn, so that the M-tiles that read the same keys are on one (16 requests of 64 tokens and 16384
    // rows 270 -> 263 us), while neighbouring pieces are on different ones (next to one another on one XCD 16 requests of one token and
    // up to 8192 rows took 54 us instead of 45).
    __device__ __forceinline__ Piece find(const Cut& c, int lane, int item) const
    {
        const int items0 = items_of(c, r), end0 = wave_scan(items0);
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
                const int in = item - of(end - items), all = c.Hkv * p.pieces;
                const int group = in / (kNumXCD * p.r.mtiles), at = in - group * (kNumXCD * p.r.mtiles);
                const int wide = min(kNumXCD, all - group * kNumXCD);
                p.mt = at / wide;
                const int head_piece = group * kNumXCD + at - p.mt * wide;
                p.kh = head_piece / p.pieces;
                p.piece = head_piece - p.kh * p.pieces;
                return p;
            }
            n0 += 64;
            if (n0 >= c.N) return p;
            const int base = __builtin_amdgcn_readlane(end, 63);
            x = {0, 0, 0, 0};
            if (n0 + lane < c.N) x = request<C>(c, n0 + lane);
            items = items_of(c, x);
            end = base + wave_scan(items);
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
    static constexpr int SW = CH < 16 ? CH - 1 : 15;     // K's swizzle repeats after 16 rows or 16 bank lines
    static constexpr int NI = T_BYTES / 1024 / WAVES;    // pieces per wavefront, tile and operand
    static constexpr int RUN = NI * RPB < 16 ? NI * RPB : 16;      // rows that are moved together: they lie in one page
    static constexpr int SLOTS = WAVES == 8 ? 4 : 2;     // of K and of V
    static constexpr bool HALF = BF16;                   // partial results in fp16
    static constexpr int COLS = HALF ? D / 16 : D / 8;   // 16-byte columns of a lane's partial results
    static constexpr int V_RING = SLOTS * T_BYTES;
    static constexpr int LDS = 2 * SLOTS * T_BYTES;
    static_assert(NI >= 1, "a tile has a piece for every wavefront");
};

// four neighbouring channels
__device__ __forceinline__ void store4(float* p, const float (&x)[4]) { *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]}; }
__device__ __forceinline__ void store4(uint16_t* p, const float (&x)[4])
{
    u32x2 w;
    w[0] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[0]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[1]) << 16;
    w[1] = (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[2]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[3]) << 16;
    *reinterpret_cast<u32x2*>(p) = w;
}

template <typename T, int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES == 4 ? 2 : 1) void attn_kernel(Args a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using C = Cfg<T, D, WAVES>;
    constexpr int KT = C::KT, DB = D / 32;
    extern __shared__ __align__(16) unsigned char lds[];
    const int tid = thread_id_x(), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
    // (two workgroups share a compute unit, and the second one's first wavefront comes to the second SIMD: where two of four wavefronts have rows,
    // they change places there, so that every SIMD has one.  fp32, 4 requests of 8 tokens, 28 / 4 heads of 128, 4096 rows 52.6 -> 38.4 us)
    const int turn = WAVES == 4 && a.used == 2 && (wg_id_x() & kNumCU) ? 3 : 0;
    const int wave = __builtin_amdgcn_readfirstlane(((tid >> 6) + turn) & (WAVES - 1));

    // ---- this workgroup's piece --------------------------------------------------------------------------------------
    Cutting<C> cutting;
    cutting.set(a.cut, lane);
    const Piece p = cutting.find(a.cut, lane, (int)wg_id_x());
    if (p.n < 0) return;
    const int n = p.n, kh = p.kh, len = p.r.len, count = p.r.count;
    const int cache_tiles = (len + KT - 1) / KT;
    // page numbers, one a lane: of an even window of 64 pages and of an odd one
    const int32_t* const table = a.table + (long long)n * a.max_pages;
    auto window_at = [&](int w) { return table[min((w << 6) + lane, a.max_pages - 1)]; };
    int t_begin, t_end;
    {
        const int each = p.r.tiles / p.pieces, more = p.r.tiles - each * p.pieces;
        t_begin = __builtin_amdgcn_readfirstlane(each * p.piece + min(p.piece, more));
        t_end = __builtin_amdgcn_readfirstlane(t_begin + each + (p.piece < more ? 1 : 0));
    }
    int window0 = (t_begin * KT >> a.page_shift) >> 6, window1 = window0;
    int entries0 = window_at(window0), entries1 = entries0;
    if (window0 & 1) window0 = -1; else window1 = -1;

    // ---- rows ----------------------------------------------------------------------------------------------------------
    const int G = a.cut.G, rows = count * G;
    const int mrows = rows_per_mtile(rows, p.r.mtiles), row0 = p.mt * mrows, row_end = min(row0 + mrows, rows);
    const int row = row0 + wave * 32 + l32;
    const bool row_ok = row < row_end;
    const bool busy = row0 + wave * 32 < row_end;      // (others move their share of the tiles)
    const int row_c = min(row, rows - 1);
    const int token = fast_div(row_c, a.cut.dG), g = row_c - token * G;
    if (a.causal) {      // keys behind the M-tile's last token are not seen
        const int last = fast_div(row_end - 1, a.cut.dG);
        t_end = min(t_end, cache_tiles + last / KT + 1);
    }
    const uint64_t* const bits = a.mask ? a.mask + n * a.mask_stride + (long long)token * ((a.cut.B + 63) >> 6) : nullptr;

    // ---- queries: B operand of S^T = K Q^T --------------------------------------------------------------------------------
    constexpr int QF = D * (int)sizeof(T) / 32;       // 16-byte fragments of a lane: half of a row
    u32x4 qf[QF];
    {
        const char* const qp = static_cast<const char*>(a.q) + (((long long)n * a.cut.B + token) * a.q_stride + (kh * G + g) * D) * (long long)sizeof(T) + half * 16;
#pragma unroll
        for (int i = 0; i < QF; ++i) qf[i] = *reinterpret_cast<const u32x4*>(qp + i * 32);
    }
    uint64_t bits0 = ~0ull;
    if (bits) bits0 = bits[0];
    // (they are here from now on: a first use behind the requests below would wait for the tiles on their way too)
#pragma unroll
    for (int i = 0; i < QF; ++i) asm volatile("" : "+v"(qf[i]));
    asm volatile("" : "+v"(bits0));
    auto in_pool = [&](int page) { return min(max(page, 0), a.pages - 1); };
    entries0 = in_pool(entries0);
    entries1 = in_pool(entries1);

    // ---- tiles: global memory -> LDS --------------------------------------------------------------------------------------
    auto page_at = [&](int index) __attribute__((always_inline)) -> int {
        const int w = index >> 6;
        if (w & 1) {
            if (w != window1) {
                window1 = w;
                entries1 = in_pool(window_at(w));      // (used here: a wait behind the branch would be one for all tiles on their way, every time)
            }
            return __builtin_amdgcn_readlane(entries1, index & 63);
        } else {
            if (w != window0) {
                window0 = w;
                entries0 = in_pool(window_at(w));
            }
            return __builtin_amdgcn_readlane(entries0, index & 63);
        }
    };
    constexpr int ROW_SHIFT = C::ROW == 512 ? 9 : C::ROW == 256 ? 8 : 7;
    const uint32_t page_bytes = (uint32_t)C::ROW << a.page_shift;
    auto page_base = [&](int page) { return (unsigned long long)((uint32_t)page * (uint32_t)a.cut.Hkv + (uint32_t)kh) << (a.page_shift + ROW_SHIFT); };
    const int page_mask = (1 << a.page_shift) - 1;
    const int row_w = wave * C::NI * C::RPB;          // first row of a tile that this wavefront moves
    const int lane_row = row_w + lane / C::CH, lane_at = lane % C::CH;
    // the 16-byte piece of row r that comes to lie at `lane_at`
    auto k_from = [&](int r) { return lane_at ^ ((r / C::RPL) & C::SW); };
    auto v_from = [&](int r) { return C::BF16 ? lane_at ^ ((((r / C::RPL) & 3) << 2) & (C::CH - 1)) : lane_at; };
    // Offsets of this lane in a run of RUN rows, which lies in one page, less what the instruction's offset adds (1 KB a piece, to
    // both sides).  They are the same for every run: the swizzles repeat after 16 rows, V's after a piece.
    uint32_t k_voff[C::RUN / C::RPB];
#pragma unroll
    for (int i = 0; i < C::RUN / C::RPB; ++i) k_voff[i] = (uint32_t)((lane / C::CH) * C::ROW + k_from(lane_row + i * C::RPB) * 16);
    const uint32_t v_voff = (uint32_t)((lane / C::CH) * C::ROW + v_from(lane_row) * 16);
    // K or V of tile t, all of whose rows are there; `pages`: where its runs' pages lie in the pools
    constexpr int RUNS = C::NI * C::RPB / C::RUN;
    auto find_pages = [&](int t, unsigned long long (&pages)[RUNS]) __attribute__((always_inline)) {
        each<0, RUNS>([&](auto run) __attribute__((always_inline)) {
            constexpr int R0 = decltype(run)::value * C::RUN;
            pages[decltype(run)::value] = page_base(page_at((t * KT + row_w + R0) >> a.page_shift));
        });
    };
    auto fetch_full = [&](auto is_v, int t, int slot, const unsigned long long (&pages)[RUNS]) __attribute__((always_inline)) {
        constexpr bool V = decltype(is_v)::value;
        unsigned char* const dst = lds + (V ? C::V_RING : 0) + slot * C::T_BYTES + wave * (C::NI * 1024);
        each<0, RUNS>([&](auto run) __attribute__((always_inline)) {
            constexpr int R0 = decltype(run)::value * C::RUN;
            const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(V ? a.v_pages : a.k_pages)) + pages[decltype(run)::value], 0, page_bytes, RSRC_FLAGS);
            const uint32_t in_page = (uint32_t)((t * KT + row_w + R0) & page_mask) * C::ROW;
            each<0, C::RUN / C::RPB>([&](auto piece) __attribute__((always_inline)) {
                constexpr int i = decltype(piece)::value;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(dst + R0 * C::ROW + i / 4 * 4096), 16, V ? v_voff : k_voff[i], in_page + i / 4 * 4096, i % 4 * 1024, 0);
            });
        });
    };
    // any tile
    auto fetch = [&](auto is_v, int t, int slot) __attribute__((always_inline)) {
        constexpr bool V = decltype(is_v)::value;
        unsigned char* const dst = lds + (V ? C::V_RING : 0) + slot * C::T_BYTES + wave * (C::NI * 1024);
        if ((t + 1) * KT <= len) {
            unsigned long long pages[RUNS];
            find_pages(t, pages);
            fetch_full(is_v, t, slot, pages);
            return;
        }
        // the last tile of the cache (what lies behind its last row is this row again), and the request's own tokens
        const bool cache = t < cache_tiles;
        const int key0 = cache ? t * KT : (t - cache_tiles) * KT, last = (cache ? len : count) - 1 - key0;
        const long long stride = cache ? D : V ? a.v_stride : a.k_stride;
#pragma unroll 1
        for (int i = 0; i < C::NI; ++i) {
            const char* base;
            int from_row = 0;
            if (cache) {      // (a piece lies in one page; one behind the last row is that row's)
                const int first = min(row_w + i * C::RPB, last);
                base = static_cast<const char*>(V ? a.v_pages : a.k_pages) + page_base(page_at((key0 + first) >> a.page_shift));
                from_row = (key0 + first) & ~page_mask;
            } else {
                base = static_cast<const char*>(V ? a.bv : a.bk) + (((long long)n * a.cut.B + key0) * stride + kh * D) * (long long)sizeof(T);
                from_row = key0;
            }
            const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, 0xffffffffu, RSRC_FLAGS);
            const int r = lane_row + i * C::RPB;
            const uint32_t at = (uint32_t)(key0 + min(r, last) - from_row) * (uint32_t)stride * (uint32_t)sizeof(T);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)(dst + i * 1024), 16, at + (V ? v_from(r) : k_from(r)) * 16, 0, 0, 0);
        }
    };
    const std::false_type is_k;
    const std::true_type is_v;

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
    constexpr int KB = KT / 32;
    // keys of tile t that the row does not see: whether there are any, and their scores out of the way
    const int first_token = fast_div(min(row0 + wave * 32, rows - 1), a.cut.dG);
    auto is_masked = [&](int t) {
        if (t < cache_tiles) return (t + 1) * KT > len;
        const int end = (t - cache_tiles + 1) * KT;
        return end > count || bits || (a.causal && end - 1 > first_token);
    };
    auto mask_scores = [&](int t, f32x16 (&s)[KB]) __attribute__((always_inline)) {
        const bool cache = t < cache_tiles;
        const int key0 = cache ? t * KT : (t - cache_tiles) * KT;
        const int valid = cache ? len - key0 : count - key0;
        uint64_t see = valid >= 64 ? ~0ull : (1ull << valid) - 1;
        if (!cache) {
            if (bits) see &= (key0 < 64 ? bits0 : bits[key0 >> 6]) >> (key0 & 63);
            else if (a.causal) see &= token - key0 >= 63 ? ~0ull : token < key0 ? 0ull : (2ull << (token - key0)) - 1;
        }
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const uint32_t w = (uint32_t)(see >> (32 * kb + 4 * half));
#pragma unroll
            for (int v = 0; v < 16; ++v) s[kb][v] = (w >> (8 * (v / 4) + v % 4)) & 1 ? s[kb][v] : -INFINITY;
        }
    };
    auto largest = [&](const f32x16 (&s)[KB]) __attribute__((always_inline)) {
        float mx = s[0][0];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[kb][v]);
        return mx;
    };

    // fragments: K's 16-byte piece 2 i + half of row l32 of a 32-key block; V's as the transposing reads take them
    const int k_off = l32 * C::ROW, k_swz = (l32 / C::RPL) & C::SW;
    constexpr int S = C::SLOTS;
    if constexpr (C::BF16) {
        // K runs a tile ahead of V: step t takes the exponentials of tile t while the matrix pipe works on the scores of t + 1,
        // then on P V of t while the vector ALUs look for the maximum of t + 1.  Requested in step t: K of t + S, V of t + S - 1.
        // (fragment i lies at the place of fragment 0 with i XORed in, as channels db of V do)
        const int k_frag = k_off + ((half ^ k_swz) << 4);
        int v_frag;
        {
            const int row_l = half * 4 + ((lane & 15) >> 2), x = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
            const int sw = (((row_l / C::RPL) & 3) << 2) & (C::CH - 1);
            v_frag = C::V_RING + row_l * C::ROW + ((x ^ sw) << 4) + (lane & 1) * 8;
        }
        auto read_k = [&](int base, auto jc) __attribute__((always_inline)) {
            constexpr int j = decltype(jc)::value;
            return *reinterpret_cast<const bf16x8*>(lds + ((base + k_frag) ^ (j % QF << 5)) + j / QF * 32 * C::ROW);
        };
        auto read_v = [&](int base, auto jc) __attribute__((always_inline)) {      // 16-key step j / DB, channels j % DB
            constexpr int j = decltype(jc)::value;
            const unsigned char* const p0 = lds + ((base + v_frag) ^ (j % DB << 6)) + j / DB * 16 * C::ROW;
            const i16x4 lo = read_tr((const lds_i16x4*)p0), hi = read_tr((const lds_i16x4*)(p0 + 8 * C::ROW));
            typedef short i16x8 __attribute__((ext_vector_type(8)));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        constexpr int NQ = 2 * QF, NP = 4 * DB;      // matrix instructions of a tile's scores and of its P V
        constexpr int AHEAD = 3;                     // fragments are read so far ahead
        const int tiles = t_end - t_begin;
        // Half tiles are requested in the order K0 V0 K1 V1 ..: `n` of them may still be on their way
        auto wait_halves = [&](int n) {
            constexpr int H = C::NI;
            if (n >= 4 && 4 * H < 64) wait_loads<4 * H < 64 ? 4 * H : 0>();
            else if (n >= 3 && 3 * H < 64) wait_loads<3 * H < 64 ? 3 * H : 0>();
            else if (n >= 2) wait_loads<2 * H>();
            else if (n == 1) wait_loads<H>();
            else wait_loads<0>();
        };
        // what the first step needs; the rest of the ring follows behind the first tile (all at once, it waited behind the others')
        if (tiles > 0) {
            fetch(is_k, t_begin, 0);
            fetch(is_v, t_begin, 0);
        }
        if (tiles > 1) fetch(is_k, t_begin + 1, 1);
        auto fill_ring = [&] {
#pragma unroll 1
            for (int i = 1; i + 1 < S && i < tiles; ++i) {
                fetch(is_v, t_begin + i, i);
                if (i + 1 < tiles) fetch(is_k, t_begin + i + 1, i + 1);
            }
        };
        // pages of the tile whose V is requested next in the steps that request whole tiles only
        unsigned long long pages[RUNS];
        float mx = -INFINITY;      // the largest score of the tile whose probabilities are next, over this lane's half of its keys
        // Step i: the probabilities of tile i (scores in s) and P V; scores of tile i + 1 into `to`.
        auto step = [&](auto next, auto whole, int i, f32x16 (&s)[2], f32x16 (&to)[2]) __attribute__((always_inline)) {
            constexpr bool NEXT = decltype(next)::value;
            if constexpr (decltype(whole)::value) {      // everything that it touches and requests are whole tiles of the cache
                wait_loads<(2 * S - 4) * C::NI>();
                wg_barrier();
            } else {
                wait_halves(min(2 * (i + S) - 1, 2 * tiles) - min(2 * i + 3, 2 * tiles));       // V of tile i, K of tile i + 1 are there
                wg_barrier();       // for everyone, and everyone is done with the slots that are requested now
                if (i + S - 1 < tiles) fetch(is_v, t_begin + i + S - 1, (i + S - 1) % S);
                if (i + S < tiles) fetch(is_k, t_begin + i + S, i % S);
            }
            const int k_base = (i + 1) % S * C::T_BYTES, v_base = i % S * C::T_BYTES;
            typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
            bf16x8 f[AHEAD + 1];
            u32x4 pw[4];         // probabilities, B operands of P V
            float mc = 0.f;
            auto read = [&](auto jc) __attribute__((always_inline)) {
                constexpr int j = decltype(jc)::value;
                if constexpr (j < NQ) return read_k(k_base, jc);
                else return read_v(v_base, std::integral_constant<int, j - NQ>());
            };
            // An exponential is taken in three stages, each beside the next one's or the one after next's: none waits for what it needs.
            auto scale = [&](auto entry) __attribute__((always_inline)) {
                constexpr int e = decltype(entry)::value;
                float x = fmaf(s[e / 16][e % 16], a.c, -mc);
                asm volatile("" : "+v"(x));
                s[e / 16][e % 16] = x;
            };
            auto tick = [&](auto tc) __attribute__((always_inline)) {
                constexpr int t = decltype(tc)::value;
                if constexpr (t < 32) {
                    float x = exp2_fast(s[t / 16][t % 16]);
                    asm volatile("" : "+v"(x));
                    s[t / 16][t % 16] = x;
                }
                SCHED_FENCE();
                if constexpr (t % 2 == 0 && t > 0) {
                    constexpr int e = t - 2;
                    const bf16x2 pair = {(__bf16)s[e / 16][e % 16], (__bf16)s[e / 16][e % 16 + 1]};
                    uint32_t w = __builtin_bit_cast(uint32_t, pair);
                    asm volatile("" : "+v"(w));
                    pw[e / 8][e / 2 % 4] = w;
                }
                if constexpr (t + 2 < 32) scale(std::integral_constant<int, t + 2>());
                SCHED_FENCE();
            };
            // tick t stands in slot t * SPAN / TICKS
            constexpr int J0 = NEXT ? 0 : NQ, TICKS = 33, SPAN = NQ + NP - DB;
            static_assert(8 * SPAN / TICKS < NQ && 16 * SPAN / TICKS < NQ + DB && 24 * SPAN / TICKS < NQ + 2 * DB && 32 * SPAN / TICKS < NQ + 3 * DB, "probabilities before their use");
            each<J0, J0 + AHEAD>([&](auto jc) __attribute__((always_inline)) { f[decltype(jc)::value % (AHEAD + 1)] = read(jc); });
            SCHED_FENCE();
            update_reference(mx);
            mc = m_ref * a.c;
            mx = -INFINITY;
            SCHED_FENCE();
            scale(std::integral_constant<int, 0>());
            scale(std::integral_constant<int, 1>());
            SCHED_FENCE();
            each<J0, NQ + NP>([&](auto jc) __attribute__((always_inline)) {
                constexpr int j = decltype(jc)::value;
                if constexpr (j + AHEAD < NQ + NP) f[(j + AHEAD) % (AHEAD + 1)] = read(std::integral_constant<int, j + AHEAD>());
                const bf16x8 x = f[j % (AHEAD + 1)];
                if constexpr (decltype(whole)::value) {      // the requests stand between the matrix instructions, whose shadow they are made in
                    if constexpr (j == NQ) fetch_full(is_v, t_begin + i + S - 1, (i + S - 1) % S, pages);
                    if constexpr (j == NQ + NP / 4) find_pages(t_begin + i + S, pages);
                    if constexpr (j == NQ + NP / 2) fetch_full(is_k, t_begin + i + S, i % S, pages);
                }
                if constexpr (!NEXT && j == NQ) each<0, (NQ * TICKS + SPAN - 1) / SPAN>(tick);
                if constexpr (j < NQ) {
                    if constexpr (j % QF) to[j / QF] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, __builtin_bit_cast(bf16x8, qf[j % QF]), to[j / QF], 0, 0, 0);
                    else to[j / QF] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, __builtin_bit_cast(bf16x8, qf[j % QF]), f32x16{}, 0, 0, 0);
                } else {
                    constexpr int jj = j - NQ;
                    o[jj % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, __builtin_bit_cast(bf16x8, pw[jj / DB]), o[jj % DB], 0, 0, 0);
                }
                SCHED_FENCE();
                each<(j * TICKS + SPAN - 1) / SPAN < TICKS ? (j * TICKS + SPAN - 1) / SPAN : TICKS, ((j + 1) * TICKS + SPAN - 1) / SPAN < TICKS ? ((j + 1) * TICKS + SPAN - 1) / SPAN : TICKS>(tick);
                if constexpr (NEXT && j >= NQ + 2) {
                    constexpr int q = j - NQ - 2;
                    each<q * 16 / (NP - 2), (q + 1) * 16 / (NP - 2)>([&](auto vc) __attribute__((always_inline)) {
                        constexpr int v = decltype(vc)::value;
                        mx = fmaxf(fmaxf(mx, to[0][v]), to[1][v]);
                        asm volatile("" : "+v"(mx));
                    });
                }
                SCHED_FENCE();
            });
            // (summed as rounded: numerator and denominator see the same values)
            const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
            float sum0 = 0.f, sum1 = 0.f;
            each<0, 8>([&](auto kc) __attribute__((always_inline)) {
                constexpr int k = 2 * decltype(kc)::value;
                sum0 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (uint32_t)pw[k / 4][k % 4]), ones, sum0, false);
                sum1 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (uint32_t)pw[k / 4][k % 4 + 1]), ones, sum1, false);
            });
            l_run += sum0 + sum1;
            if constexpr (NEXT && !decltype(whole)::value)
                if (is_masked(t_begin + i + 1)) {
                    mask_scores(t_begin + i + 1, to);
                    mx = largest(to);
                }
        };
        if (!busy) {      // the same requests, waits and barriers as below
            if (tiles > 0) {
                wait_halves(min(3, 2 * tiles) - 1);
                wg_barrier();
                fill_ring();
            }
#pragma unroll 1
            for (int i = 0; i < tiles; ++i) {
                wait_halves(min(2 * (i + S) - 1, 2 * tiles) - min(2 * i + 3, 2 * tiles));
                wg_barrier();
                if (i + S - 1 < tiles) fetch(is_v, t_begin + i + S - 1, (i + S - 1) % S);
                if (i + S < tiles) fetch(is_k, t_begin + i + S, i % S);
            }
        } else if (tiles > 0) {
            f32x16 s0[2], s1[2];
            wait_halves(min(3, 2 * tiles) - 1);      // K of the first tile
            wg_barrier();
            fill_ring();
            {
                bf16x8 f[AHEAD + 1];
                each<0, AHEAD>([&](auto jc) __attribute__((always_inline)) { f[decltype(jc)::value] = read_k(0, jc); });
                each<0, NQ>([&](auto jc) __attribute__((always_inline)) {
                    constexpr int j = decltype(jc)::value;
                    if constexpr (j + AHEAD < NQ) f[(j + AHEAD) % (AHEAD + 1)] = read_k(0, std::integral_constant<int, j + AHEAD>());
                    const bf16x8 x = f[j % (AHEAD + 1)], q = __builtin_bit_cast(bf16x8, qf[j % QF]);
                    if constexpr (j % QF) s0[j / QF] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, q, s0[j / QF], 0, 0, 0);
                    else s0[j / QF] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, q, f32x16{}, 0, 0, 0);
                });
            }
            if (is_masked(t_begin)) mask_scores(t_begin, s0);
            mx = largest(s0);
            // (two steps a round: the scores change places without moves)
            const std::true_type yes;
            const std::false_type no;
            int i = 0;
            const int whole = min(t_end, len / KT) - t_begin - S;      // steps that request whole tiles
            if (whole >= 2) find_pages(t_begin + S - 1, pages);
            for (; i + 2 <= whole; i += 2) {
                step(yes, yes, i, s0, s1);
                step(yes, yes, i + 1, s1, s0);
            }
            for (; i + 2 < tiles; i += 2) {
                step(yes, no, i, s0, s1);
                step(yes, no, i + 1, s1, s0);
            }
            if (i + 1 < tiles) {
                step(yes, no, i, s0, s1);
                step(no, no, i + 1, s1, s0);
            } else {
                step(no, no, i, s0, s1);
            }
        }
    } else {
        auto step = [&](int t, int slot) {
            const unsigned char* const kt = lds + slot * C::T_BYTES;
            const unsigned char* const vt = kt + C::V_RING;
            f32x16 s[1];
#pragma unroll
            for (int v = 0; v < 16; ++v) s[0][v] = 0.f;
#pragma unroll
            for (int i = 0; i < QF; ++i) {
                const f32x4 kx = *reinterpret_cast<const f32x4*>(kt + k_off + (((2 * i + half) ^ k_swz) << 4)), qx = __builtin_bit_cast(f32x4, qf[i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) s[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(kx[j], qx[j], s[0], 0, 0, 0);
            }
            if (is_masked(t)) mask_scores(t, s);
            update_reference(largest(s));
            const float mc = m_ref * a.c;
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                s[0][v] = exp2_fast(fmaf(s[0][v], a.c, -mc));
                sum += s[0][v];
            }
            l_run += sum;
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const unsigned char* const vp = vt + (8 * (v / 4) + 4 * half + v % 4) * C::ROW + l32 * 4;
#pragma unroll
                for (int db = 0; db < DB; ++db)
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(*reinterpret_cast<const float*>(vp + db * 128), s[0][v], o[db], 0, 0, 0);
            }
        };
#pragma unroll
        for (int i = 0; i < S - 1; ++i)
            if (t_begin + i < t_end) {
                fetch(is_k, t_begin + i, i);
                fetch(is_v, t_begin + i, i);
            }
        int slot = 0;
        for (int t = t_begin; t < t_end; ++t) {
            wait_loads<0>();
            wg_barrier();       // the tile is there, and everyone is done with the slot that the next one goes to
            if (t + S - 1 < t_end) {
                fetch(is_k, t + S - 1, slot == 0 ? S - 1 : slot - 1);
                fetch(is_v, t + S - 1, slot == 0 ? S - 1 : slot - 1);
            }
            if (busy) step(t, slot);
            slot = slot + 1 == S ? 0 : slot + 1;
        }
    }

    // ---- out ---------------------------------------------------------------------------------------------------------------
    const float l = l_run + other_half(l_run);      // (0: the row sees nothing.  Where fp32 calls have a NaN here, the row becomes NaN)
    // Partial results go through the L2s to memory (aux 16: device scope): the merge's wavefronts are on other XCDs, and what is left
    // dirty goes out only when the launch has ended (4 requests of 32 tokens, 4096 rows 24.1 -> 23.3 us; 16 of a token, whose stores are parts of lines,
    // 40.4 -> 40.8: a branch for these cost as much).
    const long long place = (long long)p.item * a.used + wave;
    constexpr int O_BYTES = DB * (C::HALF ? 2 : 4) * 1024;
    const __amdgpu_buffer_rsrc_t o_rsrc = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<char*>(a.ws_o) + place * O_BYTES, 0, O_BYTES, RSRC_FLAGS);
    const __amdgpu_buffer_rsrc_t ml_rsrc = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<char*>(a.ws_ml) + place * 512, 0, 512, RSRC_FLAGS);
    auto put = [](const __amdgpu_buffer_rsrc_t& rsrc, int at, u32x4 w) __attribute__((always_inline)) { __builtin_amdgcn_raw_buffer_store_b128(w, rsrc, at, 0, 16); };
    if (p.pieces == 1) {
        if (!row_ok) return;
        const float inv = l == 0.f ? 0.f : 1.f / l;
        T* const op = static_cast<T*>(a.out) + (((long long)n * a.cut.B + token) * a.Hq + kh * G + g) * D + 4 * half;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int v4 = 0; v4 < 4; ++v4) {
                float x[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = l == 0.f ? 0.f : o[db][4 * v4 + j] * inv;
                store4(op + db * 32 + v4 * 8, x);
            }
    } else if constexpr (C::HALF) {
        // averages in fp16, times a power of two that brings the row's largest to 2^14 .. 2^15
        const float inv = l == 0.f ? 0.f : 1.f / l;
        float top = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                o[db][v] *= inv;
                top = fmaxf(top, __builtin_fabsf(o[db][v]));
            }
        top = fmaxf(top, other_half(top));
        const int up = max(min(14 + 127 - (int)(__builtin_bit_cast(uint32_t, top) >> 23 & 255u), 126), -126);
        const float scale = __builtin_bit_cast(float, (uint32_t)(127 + up) << 23), back = __builtin_bit_cast(float, (uint32_t)(127 - up) << 23);
        if (!row_ok) return;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                f16x8 w;
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = (_Float16)(o[db][8 * c + j] * scale);
                put(o_rsrc, (db * 2 + c) * 1024 + lane * 16, __builtin_bit_cast(u32x4, w));
            }
        if (half == 0) put(ml_rsrc, l32 * 16, __builtin_bit_cast(u32x4, f32x4{l == 0.f ? -INFINITY : m_ref * a.c, l, back, 0.f}));
    } else if (row_ok) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int v4 = 0; v4 < 4; ++v4)
                put(o_rsrc, (db * 4 + v4) * 1024 + lane * 16, __builtin_bit_cast(u32x4, f32x4{o[db][4 * v4], o[db][4 * v4 + 1], o[db][4 * v4 + 2], o[db][4 * v4 + 3]}));
        if (half == 0) put(ml_rsrc, l32 * 16, __builtin_bit_cast(u32x4, f32x4{l == 0.f ? -INFINITY : m_ref * a.c, l, 1.f, 0.f}));
    }
#endif
}

struct MergeArgs {
    Cut cut;
    const float* ws_o;
    const float* ws_ml;
    void* out;
    int Hq, max_mt, used;
};

// One wavefront, or SPLIT of them, per (request, KV head, M-tile, its 32-row wavefront, 16-byte column): lane = as in the accumulators.  Bound by
// latency: up to 16 pieces are on their way at a time, and there are as many wavefronts as columns.  16 requests of one token and up to 8192 rows
// 5.5 us; one of 32768 rows, 103 pieces a KV head, 7.4.
template <typename T, int D, int WAVES, int SPLIT>
__global__ __launch_bounds__(256) void merge_kernel(MergeArgs a)
{
#if defined(__HIP_DEVICE_COMPILE__)
    using C = Cfg<T, D, WAVES>;
    constexpr int COLS = C::COLS;
    const int tid = thread_id_x(), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
    const int share = SPLIT > 1 ? __builtin_amdgcn_readfirstlane(tid >> 6) : 0;
    int job = SPLIT > 1 ? (int)wg_id_x() : __builtin_amdgcn_readfirstlane((int)wg_id_x() * 4 + (tid >> 6));
    const int col = job % COLS;
    job /= COLS;
    const int wave = job % a.used, mtile = job / a.used;
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
    const int rows = mine.count * a.cut.G, mrows = rows_per_mtile(rows, mine.mtiles);
    const int row = mt * mrows + wave * 32 + l32;
    if (wave * 32 >= mrows || mt * mrows + wave * 32 >= rows) return;
    const bool row_ok = row < min((mt + 1) * mrows, rows);
    if (SPLIT == 1 && !row_ok) return;
    const int all = a.cut.Hkv * pieces;
    // item of piece i: see Cutting::find
    auto item_of = [&](int i) {
        const int head_piece = kh * pieces + i, group = head_piece / kNumXCD, wide = min(kNumXCD, all - group * kNumXCD);
        return (long long)(base + group * kNumXCD * mine.mtiles + mt * wide + head_piece - group * kNumXCD);
    };
    typedef std::conditional_t<C::HALF, f16x8, f32x4> Part;
    constexpr int E = 16 / sizeof(Part{}[0]);
    const f32x4* const ml0 = reinterpret_cast<const f32x4*>(a.ws_ml) + wave * 32 + l32;
    const Part* const wo0 = reinterpret_cast<const Part*>(a.ws_o) + (wave * COLS + col) * 64 + lane;
    float m = -INFINITY, l_sum = 0.f, y[E];
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = 0.f;
    const int first = pieces * share / SPLIT, last = pieces * (share + 1) / SPLIT, mine_all = last - first;
    auto join = [&](auto unroll) __attribute__((always_inline)) {
        constexpr int UNROLL = decltype(unroll)::value;
        for (int i = first; i < last; i += UNROLL) {
            f32x4 ml[UNROLL];
            Part w[UNROLL];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const long long at = item_of(min(i + u, last - 1));
                ml[u] = ml0[at * (a.used * 32)];
                w[u] = wo0[at * (a.used * COLS * 64)];
            }
            // (all of them are requested before the first is awaited)
            SCHED_FENCE();
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                u32x4 x = __builtin_bit_cast(u32x4, w[u]);
                asm volatile("" : "+v"(ml[u]), "+v"(x));
                w[u] = __builtin_bit_cast(Part, x);
            }
            float top = m;
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                if (i + u >= last) ml[u][0] = -INFINITY;
                top = fmaxf(top, ml[u][0]);
            }
            const float ref = top == -INFINITY ? 0.f : top;
            const float old = exp2_fast(m - ref);
            m = top;
            l_sum *= old;
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] *= old;
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const float f = exp2_fast(ml[u][0] - ref);
                l_sum = fmaf(f, ml[u][1], l_sum);
                // (averages count with the sum that they are of; a piece that the row sees nothing of is 0)
                const float g = C::HALF ? f * ml[u][1] * ml[u][2] : f;
#pragma unroll
                for (int e = 0; e < E; ++e) y[e] = fmaf(g, (float)w[u][e], y[e]);
            }
        }
    };
    if (mine_all <= 2) join(std::integral_constant<int, 2>());
    else if (mine_all <= 4) join(std::integral_constant<int, 4>());
    else if (mine_all <= 8) join(std::integral_constant<int, 8>());
    else join(std::integral_constant<int, 16>());
    if constexpr (SPLIT > 1) {
        // the wavefronts' shares, in their order
        __shared__ float s_m[SPLIT][64], s_l[SPLIT][64], s_y[SPLIT][E][64];
        s_m[share][lane] = m;
        s_l[share][lane] = l_sum;
#pragma unroll
        for (int e = 0; e < E; ++e) s_y[share][e][lane] = y[e];
        __syncthreads();
        if (share || !row_ok) return;
        float top = m;
#pragma unroll
        for (int w = 1; w < SPLIT; ++w) top = fmaxf(top, s_m[w][lane]);
        const float ref = top == -INFINITY ? 0.f : top, own = exp2_fast(m - ref);
        l_sum *= own;
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] *= own;
#pragma unroll
        for (int w = 1; w < SPLIT; ++w) {
            const float x = exp2_fast(s_m[w][lane] - ref);
            l_sum = fmaf(x, s_l[w][lane], l_sum);
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = fmaf(x, s_y[w][e][lane], y[e]);
        }
    }
    const int token = fast_div(row, a.cut.dG), g = row - token * a.cut.G;
    const float inv = l_sum == 0.f ? 0.f : 1.f / l_sum;
    T* const op = static_cast<T*>(a.out) + (((long long)n * a.cut.B + token) * a.Hq + kh * a.cut.G + g) * D + 4 * half + col * (2 * E);
#pragma unroll
    for (int c = 0; c < E / 4; ++c) {
        float z[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = l_sum == 0.f ? 0.f : y[4 * c + e] * inv;
        store4(op + 8 * c, z);
    }
#endif
}

// ---- host ----------------------------------------------------------------------------------------------------------------

struct Plan {
    int waves, used, kt, max_mt, W;
    int max_len;
    long long items;            // no call has more pieces
    bool partials;              // some request may have more than one piece
    size_t o_bytes, ml_bytes;
};

inline Plan make_plan(const fdd_paged_cache& c, const fdd_paged_attn_params& p)
{
    Plan pl;
    const long long rows = (long long)p.B * (p.Hq / c.Hkv);
    // Four wavefronts up to 128 rows, and up to 256 where there are few (request, KV head) pairs: more, shorter pieces start sooner than keys are brought
    // twice (us, 4 wavefronts and 8: 8 requests of 224 rows, 2048 keys 23.6 and 24.8, 4 of 4096 24.4 and 25.2; 16 of 16384 150 and 145, 64 of 2048 100 and 87; numbers of
    // requests whose pieces are W and no more in either form).
    pl.waves = rows <= 128 || (rows <= 256 && c.N * c.Hkv <= 32) || c.dtype == FDD_F32 ? 4 : 8;
    pl.used = rows < pl.waves * 32 ? (int)((rows + 31) / 32) : pl.waves;
    pl.kt = c.dtype == FDD_BF16 ? 64 : 32;
    const int capacity = c.max_pages * c.page_size;
    pl.max_len = p.max_len > 0 ? (p.max_len < capacity ? p.max_len : capacity) : capacity;
    pl.max_mt = (int)((rows + pl.waves * 32 - 1) / (pl.waves * 32));
    pl.W = pl.waves == 8 ? kNumCU : 2 * kNumCU;
    const long long tiles = (pl.max_len + pl.kt - 1) / pl.kt + (p.B + pl.kt - 1) / pl.kt;
    const long long mtiles = (long long)c.N * c.Hkv * pl.max_mt;
    pl.partials = tiles > MIN_TILES;
    pl.items = mtiles + (pl.partials ? pl.W : 0);
    const size_t prow = pl.partials ? (size_t)pl.items * pl.used * 32 : 0;
    pl.o_bytes = (prow * c.D * (c.dtype == FDD_BF16 ? 2 : 4) + 255) & ~(size_t)255;
    pl.ml_bytes = (prow * 16 + 255) & ~(size_t)255;
    return pl;
}

inline Cut make_cut(const fdd_paged_cache& c, const fdd_paged_attn_params& p, const Plan& pl)
{
    return {c.lens, p.n_tokens, c.N, p.B, p.Hq / c.Hkv, c.Hkv, make_fastdiv((uint32_t)(p.Hq / c.Hkv)), pl.max_len, pl.W};
}

template <typename T, int D, int WAVES>
hipError_t launch(const fdd_paged_cache& c, const fdd_paged_attn_params& p, const Plan& pl, const Args& a)
{
    using C = Cfg<T, D, WAVES>;
    const hipStream_t s = static_cast<hipStream_t>(p.stream);
    // the LDS limit of this instantiation is raised once per device (bit d of `done`: device d)
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (!(done.load(std::memory_order_acquire) & bit)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(attn_kernel<T, D, WAVES>), hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
        if (e != hipSuccess) return e;
        done.fetch_or(bit, std::memory_order_release);
    }
    attn_kernel<T, D, WAVES><<<dim3((unsigned)pl.items), WAVES * 64, C::LDS, s>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess || !pl.partials) return e;
    MergeArgs m = {a.cut, a.ws_o, a.ws_ml, p.out, p.Hq, pl.max_mt, pl.used};
    const long long mtiles = (long long)c.N * c.Hkv * pl.max_mt, jobs = mtiles * pl.used * C::COLS, pieces = pl.W / mtiles;
    // A request's many pieces: four wavefronts a job (one request of a token and 32768 rows, 103 pieces a KV head, 32.7 -> 22.7 us; 16 wavefronts
    // 23.7; 4 requests of 32 tokens, 13 pieces, 24.8 and 26.0)
    if (pieces < 24) merge_kernel<T, D, WAVES, 1><<<dim3((unsigned)((jobs + 3) / 4)), 256, 0, s>>>(m);
    else merge_kernel<T, D, WAVES, 4><<<dim3((unsigned)jobs), 256, 0, s>>>(m);
    return hipGetLastError();
}

// (paged_attn_f32.hip: a file of its own, which NaN passes through)
hipError_t launch_f32(const fdd_paged_cache& c, const fdd_paged_attn_params& p, const Plan& pl, const Args& a);

}  // namespace paged_attn
}  // namespace fdd
