// Attention over a paged cache (paged_attn.h): bf16, and the entry points.
#include "paged_attn.h"

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
    if (p->B > (1 << 24) || p->Hq > 65535 || tokens >= (1ll << 30) || tokens * p->Hq >= (1ll << 30)) return fail(FDD_ERR_SHAPE, "%s: N*B*Hq too large", kFn);
    const Plan pl = make_plan(*c, *p);
    const long long tiles = (pl.max_len + pl.kt - 1) / pl.kt + (p->B + pl.kt - 1) / pl.kt;
    if ((long long)c->N * c->Hkv * pl.max_mt * tiles >= (1ll << 31) - pl.W || pl.items >= (1ll << 22))
        return fail(FDD_ERR_SHAPE, "%s: N*B*Hq*max_len too large", kFn);
    // (a launch has at most 2^32 threads: the merge has a wavefront for 32 rows' four channels or eight)
    if (pl.partials && (long long)c->N * c->Hkv * pl.max_mt * pl.used * (c->D / 8) >= (1ll << 26)) return fail(FDD_ERR_SHAPE, "%s: N*B*Hq too large", kFn);
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
    if (p->mask && p->mask_stride != 0 && (p->mask_stride < words || p->mask_stride > (1ll << 56) / c->N))
        return fail(FDD_ERR_SHAPE, "%s: mask_stride=%lld must be 0 or at least %lld words, and N times it at most 2^56", kFn, (long long)p->mask_stride, words);
    const Plan pl = make_plan(*c, *p);
    Args a = {};
    a.q_stride = token_stride(p->q_stride, q_token); a.k_stride = token_stride(p->k_stride, kv_token); a.v_stride = token_stride(p->v_stride, kv_token);
    const unsigned long long out_bytes = (unsigned long long)(tokens * q_token * es), pool = pool_bytes(*c);
    const size_t need = pl.o_bytes + pl.ml_bytes;
    if (need > 0) {
        if (!p->workspace) return fail(FDD_ERR_WORKSPACE, "%s: workspace is NULL, %zu bytes needed", kFn, need);
        if (!aligned_to(p->workspace, 256)) return fail(FDD_ERR_WORKSPACE, "%s: workspace must be 256-byte aligned", kFn);
        if (p->workspace_bytes < need) return fail(FDD_ERR_WORKSPACE, "%s: workspace has %zu bytes, %zu needed", kFn, p->workspace_bytes, need);
    }
    const Span outs[] = {{p->out, out_bytes}, {need > 0 ? p->workspace : nullptr, need}};
    const Span ins[] = {{p->q, (unsigned long long)(((tokens - 1) * a.q_stride + q_token) * es)}, {p->block_k, (unsigned long long)(((tokens - 1) * a.k_stride + kv_token) * es)},
                        {p->block_v, (unsigned long long)(((tokens - 1) * a.v_stride + kv_token) * es)}, {c->k, pool}, {c->v, pool},
                        {c->page_table, (unsigned long long)c->N * c->max_pages * 4}, {c->lens, (unsigned long long)c->N * 4},
                        {p->mask, (unsigned long long)((c->N - 1) * p->mask_stride + words) * 8}, {p->n_tokens, (unsigned long long)c->N * 4}};
    if (outputs_overlap(outs, ins)) return fail(FDD_ERR_UNSUPPORTED, "%s: out or the workspace overlaps another array", kFn);
    const float scale = p->scale > 0.f ? p->scale : 1.f / std::sqrt((float)c->D);
    a.cut = make_cut(*c, *p, pl);
    a.q = p->q; a.bk = p->block_k; a.bv = p->block_v; a.k_pages = c->k; a.v_pages = c->v; a.table = c->page_table; a.mask = p->mask; a.out = p->out;
    a.ws_o = static_cast<float*>(p->workspace);
    a.ws_ml = reinterpret_cast<float*>(static_cast<char*>(p->workspace) + pl.o_bytes);
    a.mask_stride = p->mask_stride;
    a.used = pl.used;
    a.pages = c->pages; a.page_shift = __builtin_ctz((unsigned)c->page_size); a.max_pages = c->max_pages; a.Hq = p->Hq;
    a.causal = (p->flags & FDD_ATTN_CAUSAL_BLOCK) != 0;
    a.c = scale * 1.4426950408889634f;
    a.slack = 8.f / a.c;
    hipError_t e;
    if (c->dtype == FDD_F32) e = launch_f32(*c, *p, pl, a);
    else if (pl.waves == 8) e = c->D == 128 ? launch<uint16_t, 128, 8>(*c, *p, pl, a) : launch<uint16_t, 64, 8>(*c, *p, pl, a);
    else e = c->D == 128 ? launch<uint16_t, 128, 4>(*c, *p, pl, a) : launch<uint16_t, 64, 4>(*c, *p, pl, a);
    if (e != hipSuccess) return fail(FDD_ERR_LAUNCH, "%s: launch failed: %s", kFn, hipGetErrorString(e));
    return FDD_OK;
}

}  // extern "C"
