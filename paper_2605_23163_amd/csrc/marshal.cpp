// Arguments of the two calls of a denoise step, of a fork, and of the calls on a prefix cache in 8 bits, on log probabilities, on a
// paged cache and on trees of drafted tokens, from tensors to the C structs of fdd.h.
//
// Host code, a CPython module: each function but `fork` checks shapes, types and placement as binding.py and paged.py do and fills the
// struct at the given address.  It returns True, or False (and set no exception) for anything that is not the ordinary
// case - a wrong shape, a tensor subclass, an active torch function mode - and binding.py's own checks then accept it or
// raise their errors.  Nothing is kept between calls.  In Python a tensor property costs about 0.1 us, and a call reads
// 40 to 60 of them: 2.3 us for attention, 4.5 us for unmasking, beside 2.5 us per kernel launch.
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/version.h>

#include <climits>

#include "fdd.h"

namespace {

struct NotOrdinary {};

void need(bool ok)
{
    if (!ok) throw NotOrdinary();
}

const at::Tensor& tensor(PyObject* o)
{
    need(THPVariable_CheckExact(o));
    const at::Tensor& t = THPVariable_Unpack(o);
    need(t.defined() && t.layout() == at::kStrided && t.has_storage() && !t.unsafeGetTensorImpl()->has_symbolic_sizes_strides());
    return t;
}

void* pointer(const at::Tensor& t)
{
    need(t.is_cuda() && t.is_contiguous());
    return t.data_ptr();
}

void* pointer_or_null(PyObject* o) { return o == Py_None ? nullptr : pointer(tensor(o)); }

int32_t int32_of(int64_t x)
{
    need(x >= 0 && x <= INT32_MAX);
    return (int32_t)x;
}

int32_t int32_of(PyObject* o)
{
    need(PyLong_CheckExact(o));
    int over = 0;
    const long x = PyLong_AsLongAndOverflow(o, &over);
    need(!over && x >= INT32_MIN && x <= INT32_MAX);
    return (int32_t)x;
}

float float_of(PyObject* o)
{
    need(PyFloat_CheckExact(o) || PyLong_CheckExact(o));
    const double x = PyFloat_AsDouble(o);
    need(!PyErr_Occurred());
    return (float)x;
}

int dtype_code(const at::Tensor& t)
{
    if (t.scalar_type() == at::kBFloat16) return FDD_BF16;
    need(t.scalar_type() == at::kFloat);
    return FDD_F32;
}

// q, prefix_k, prefix_v, block_k, block_v, scaffold_mask, out, prefix_v_packed, ext_k, ext_v, q_positions, E, causal_block,
// splits, scale
void fill_attn(fdd_attn_params* p, PyObject* const* a)
{
    const at::Tensor &q = tensor(a[0]), &pk = tensor(a[1]), &pv = tensor(a[2]), &bk = tensor(a[3]), &bv = tensor(a[4]);
    need(q.dim() == 4 && pk.dim() == 3 && bk.dim() == 4);
    const int64_t N = q.size(0), B = q.size(1), Hkv = bk.size(2), D = q.size(3);
    need(pk.size(1) == Hkv && pk.size(2) == D && pv.sizes() == pk.sizes());
    need(bk.size(0) == N && bk.size(1) == B && bk.size(3) == D && bv.sizes() == bk.sizes());
    const auto type = q.scalar_type();
    need(pk.scalar_type() == type && pv.scalar_type() == type && bk.scalar_type() == type && bv.scalar_type() == type);
    p->N = int32_of(N); p->B = int32_of(B); p->L = int32_of(pk.size(0));
    p->Hq = int32_of(q.size(2)); p->Hkv = int32_of(Hkv); p->D = int32_of(D);
    p->dtype = (decltype(p->dtype))dtype_code(q);
    p->scale = a[14] == Py_None ? 0.f : float_of(a[14]);
    p->q = pointer(q);
    if (p->L > 0) { p->prefix_k = pointer(pk); p->prefix_v = pointer(pv); }
    p->block_k = pointer(bk); p->block_v = pointer(bv);
    p->scaffold_mask = (decltype(p->scaffold_mask))pointer_or_null(a[5]);
    p->out = pointer_or_null(a[6]);
    p->prefix_v_packed = pointer_or_null(a[7]);
    if (a[8] != Py_None) {
        const at::Tensor &ek = tensor(a[8]), &ev = tensor(a[9]);
        need(ek.dim() == 4 && ek.size(0) == N && ek.size(2) == Hkv && ek.size(3) == D && ev.sizes() == ek.sizes());
        need(ek.scalar_type() == type && ev.scalar_type() == type);
        p->ext_k = pointer(ek); p->ext_v = pointer(ev); p->ext_capacity = int32_of(ek.size(1));
    }
    if (a[10] != Py_None) {
        const at::Tensor& qp = tensor(a[10]);
        need(qp.scalar_type() == at::kInt && qp.dim() == 1);
        p->q_positions = (decltype(p->q_positions))pointer(qp);
        p->n_q_positions = int32_of(qp.numel());
    }
    p->E = int32_of(a[11]);
    const int causal = PyObject_IsTrue(a[12]);
    need(causal >= 0);
    p->flags = causal ? FDD_ATTN_CAUSAL_BLOCK : 0;
    p->splits = int32_of(a[13]);
}

// logits, mask, scaffold_mask, tokens, confidences, n_unmasked, committed, tau, refresh
void fill_unmask(fdd_unmask_params* p, PyObject* const* a)
{
    const at::Tensor &x = tensor(a[0]), &mask = tensor(a[1]), &tok = tensor(a[3]);
    need(x.dim() == 3);
    const int64_t N = x.size(0), B = x.size(1);
    auto per_position = [&](const at::Tensor& t, at::ScalarType type) {
        need(t.scalar_type() == type && t.dim() == 2 && t.size(0) == N && t.size(1) == B);
    };
    per_position(mask, at::kByte);
    per_position(tok, at::kInt);
    if (a[2] != Py_None) per_position(tensor(a[2]), at::kByte);
    p->N = int32_of(N); p->B = int32_of(B); p->V = x.size(2);
    p->dtype = (decltype(p->dtype))dtype_code(x);
    p->tau = float_of(a[7]);
    p->logits = pointer(x);
    p->mask = (decltype(p->mask))pointer(mask);
    p->scaffold_mask = (decltype(p->scaffold_mask))pointer_or_null(a[2]);
    p->tokens = (decltype(p->tokens))pointer(tok);
    p->confidences = (decltype(p->confidences))pointer_or_null(a[4]);
    p->n_unmasked = (decltype(p->n_unmasked))pointer_or_null(a[5]);
    p->committed = (decltype(p->committed))pointer_or_null(a[6]);
    if (a[8] != Py_None) {
        need(PyTuple_CheckExact(a[8]) && PyTuple_GET_SIZE(a[8]) == 4);
        auto item = [&](int i) -> const at::Tensor& { return tensor(PyTuple_GET_ITEM(a[8], i)); };
        const at::Tensor &tk = item(0), &tv = item(1), &bk = item(2), &bv = item(3);
        need(tk.dim() == 3 && bk.dim() == 4 && bk.size(0) == N && bk.size(1) == B);
        need(tk.size(1) == bk.size(2) && tk.size(2) == bk.size(3) && tv.sizes() == tk.sizes() && bv.sizes() == bk.sizes());
        p->refresh_table_k = pointer(tk); p->refresh_table_v = pointer(tv);
        p->refresh_block_k = pointer(bk); p->refresh_block_v = pointer(bv);
        p->refresh_T = int32_of(tk.size(0)); p->refresh_Hkv = int32_of(tk.size(1)); p->refresh_D = int32_of(tk.size(2));
        p->refresh_dtype = (decltype(p->refresh_dtype))dtype_code(tk);
    }
}

struct QuantCall {
    fdd_quant_cache cache;
    fdd_quant_rows rows;
};

struct AttnQuantCall {
    fdd_attn_params p;
    fdd_quant_cache cache;
};

// the tensors of these calls have to be on the current device, which Python names
struct OnDevice {
    int64_t device;
    const at::Tensor& operator()(PyObject* o) const
    {
        const at::Tensor& t = tensor(o);
        need(t.is_cuda() && t.get_device() == device);
        return t;
    }
    void* or_null(PyObject* o) const { return o == Py_None ? nullptr : pointer((*this)(o)); }
};

void fill_cache(fdd_quant_cache* c, PyObject* o, const OnDevice& on)
{
    need(PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 4);
    const at::Tensor &k = on(PyTuple_GET_ITEM(o, 0)), &v = on(PyTuple_GET_ITEM(o, 1)), &ks = on(PyTuple_GET_ITEM(o, 2)), &vs = on(PyTuple_GET_ITEM(o, 3));
    need(k.dim() == 3 && v.sizes() == k.sizes() && k.size(1) % FDD_QUANT_BLOCK == 0);
    need(ks.dim() == 2 && ks.size(0) == k.size(0) && ks.size(1) == k.size(1) / FDD_QUANT_BLOCK && vs.sizes() == ks.sizes());
    need(k.scalar_type() == at::kFloat8_e4m3fn && v.scalar_type() == at::kFloat8_e4m3fn && ks.scalar_type() == at::kFloat && vs.scalar_type() == at::kFloat);
    c->k = pointer(k); c->v = pointer(v);
    c->k_scale = (float*)pointer(ks); c->v_scale = (float*)pointer(vs);
    c->Hkv = int32_of(k.size(0)); c->capacity = int32_of(k.size(1)); c->D = int32_of(k.size(2));
}

// k, v, prefix, row0, device
void fill_quant(QuantCall* c, PyObject* const* a)
{
    const OnDevice on{int32_of(a[4])};
    const at::Tensor &k = on(a[0]), &v = on(a[1]);
    fill_cache(&c->cache, a[2], on);
    need(k.dim() == 3 && v.sizes() == k.sizes() && k.size(1) == c->cache.Hkv && k.size(2) == c->cache.D && v.scalar_type() == k.scalar_type());
    need(k.is_contiguous() && v.is_contiguous());      // (rows that lie apart are looked at in Python)
    c->rows.rows = int32_of(k.size(0));
    c->rows.dtype = (decltype(c->rows.dtype))dtype_code(k);
    const int32_t row0 = int32_of(a[3]);
    need(row0 >= 0 && row0 <= c->cache.capacity - c->rows.rows);
    c->rows.k = k.data_ptr(); c->rows.v = v.data_ptr();
    if (c->rows.rows > 1) { c->rows.k_row_stride = k.stride(0); c->rows.v_row_stride = v.stride(0); }
}

// q, prefix, L, block_k, block_v, scaffold_mask, out, ext_k, ext_v, q_positions, E, causal_block, splits, scale, device
void fill_attn_quant(AttnQuantCall* c, PyObject* const* a)
{
    const OnDevice on{int32_of(a[14])};
    const at::Tensor &q = on(a[0]), &bk = on(a[3]), &bv = on(a[4]);
    fill_cache(&c->cache, a[1], on);
    need(q.dim() == 4 && bk.dim() == 4);
    const int64_t N = q.size(0), B = q.size(1), Hkv = bk.size(2), D = q.size(3);
    need(bk.size(0) == N && bk.size(1) == B && bk.size(3) == D && bv.sizes() == bk.sizes());
    need(c->cache.Hkv == Hkv && c->cache.D == D);
    const auto type = q.scalar_type();
    need(bk.scalar_type() == type && bv.scalar_type() == type);
    fdd_attn_params* const p = &c->p;
    p->N = int32_of(N); p->B = int32_of(B); p->L = int32_of(a[2]);
    need(p->L >= 0 && p->L <= c->cache.capacity);
    p->Hq = int32_of(q.size(2)); p->Hkv = int32_of(Hkv); p->D = int32_of(D);
    p->dtype = (decltype(p->dtype))dtype_code(q);
    p->scale = a[13] == Py_None ? 0.f : float_of(a[13]);
    p->q = pointer(q);
    p->block_k = pointer(bk); p->block_v = pointer(bv);
    p->scaffold_mask = (decltype(p->scaffold_mask))on.or_null(a[5]);
    const at::Tensor& out = on(a[6]);
    need(out.sizes() == q.sizes() && out.scalar_type() == type);
    p->out = pointer(out);
    if (a[7] != Py_None) {
        const at::Tensor &ek = on(a[7]), &ev = on(a[8]);
        need(ek.dim() == 4 && ek.size(0) == N && ek.size(2) == Hkv && ek.size(3) == D && ev.sizes() == ek.sizes());
        need(ek.scalar_type() == type && ev.scalar_type() == type);
        p->ext_k = pointer(ek); p->ext_v = pointer(ev); p->ext_capacity = int32_of(ek.size(1));
    }
    if (a[9] != Py_None) {
        const at::Tensor& qp = on(a[9]);
        need(qp.scalar_type() == at::kInt && qp.dim() == 1 && qp.numel() > 0);
        p->q_positions = (decltype(p->q_positions))pointer(qp);
        p->n_q_positions = int32_of(qp.numel());
    }
    p->E = int32_of(a[10]);
    const int causal = PyObject_IsTrue(a[11]);
    need(causal >= 0);
    p->flags = causal ? FDD_ATTN_CAUSAL_BLOCK : 0;
    p->splits = int32_of(a[12]);
}

// logits, tokens, mask, top, temperature, logprobs, entropy, top_ids, top_logprobs, device
void fill_logprobs(fdd_logprob_params* p, PyObject* const* a)
{
    const OnDevice on{int32_of(a[9])};
    const at::Tensor &x = on(a[0]);
    need(x.dim() == 3);
    const int64_t N = x.size(0), B = x.size(1);
    p->N = int32_of(N); p->B = int32_of(B); p->V = x.size(2);
    p->dtype = (decltype(p->dtype))dtype_code(x);
    p->top = int32_of(a[3]);
    need(p->top >= 0 && p->top <= FDD_LOGPROBS_MAX_TOP);
    p->temperature = float_of(a[4]);
    auto per_position = [&](PyObject* o, at::ScalarType type, bool top) {
        const at::Tensor& t = on(o);
        need(t.scalar_type() == type && t.dim() == (top ? 3 : 2) && t.size(0) == N && t.size(1) == B && (!top || t.size(2) == p->top));
        return pointer(t);
    };
    p->logits = pointer(x);
    p->tokens = (decltype(p->tokens))per_position(a[1], at::kInt, false);
    if (a[2] != Py_None) p->row_mask = (decltype(p->row_mask))per_position(a[2], at::kByte, false);
    p->logprobs = (float*)per_position(a[5], at::kFloat, false);
    p->entropy = (float*)per_position(a[6], at::kFloat, false);
    void* const ids = per_position(a[7], at::kInt, true);
    void* const top = per_position(a[8], at::kFloat, true);
    if (p->top > 0) {
        p->top_ids = (decltype(p->top_ids))ids;
        p->top_logprobs = (float*)top;
    }
}

// ---- a paged cache and trees of drafted tokens -----------------------------------------------------------------------------

struct AppendCall {
    fdd_paged_cache cache;
    fdd_paged_append_params p;
    fdd_rope_table table;
};

struct PagedAttnCall {
    fdd_paged_cache cache;
    fdd_paged_attn_params p;
};

// a dense array of this type and shape, or nullptr for None
template <typename P>
P* shaped(const OnDevice& on, PyObject* o, at::ScalarType type, at::IntArrayRef shape)
{
    if (o == Py_None) return nullptr;
    const at::Tensor& t = on(o);
    need(t.scalar_type() == type && t.sizes() == shape);
    return (P*)pointer(t);
}

// the same for each of N requests, or (without that dimension) one for all of them; the entries between requests
template <typename P>
P* per_request(const OnDevice& on, PyObject* o, at::ScalarType type, int64_t N, at::IntArrayRef tail, int64_t* stride)
{
    if (o == Py_None) return nullptr;
    const at::Tensor& t = on(o);
    const bool own = t.dim() == (int64_t)tail.size() + 1;
    need(t.scalar_type() == type && (own ? t.size(0) == N && t.sizes().slice(1) == tail : t.sizes() == tail));
    if (own) {
        *stride = 1;
        for (const int64_t x : tail) *stride *= x;
    }
    return (P*)pointer(t);
}

// rows [..,heads,D] that are evenly spaced over all dimensions in front: address, and the stride of rows (0: there is one)
void* even_rows(const at::Tensor& t, int64_t* stride)
{
    const int64_t d = t.dim();
    need(d >= 2 && t.is_cuda() && t.numel() > 0);
    const int64_t H = t.size(d - 2), D = t.size(d - 1);
    need((D == 1 || t.stride(d - 1) == 1) && (H == 1 || t.stride(d - 2) == D));
    int64_t step = 0, rows = 1;
    for (int64_t i = d - 3; i >= 0; --i) {
        if (t.size(i) == 1) continue;
        need(rows == 1 || t.stride(i) == step * rows);
        if (rows == 1) step = t.stride(i);
        rows *= t.size(i);
    }
    need(rows == 1 || step >= H * D);
    *stride = step;
    return t.data_ptr();
}

void fill_table(fdd_rope_table* r, PyObject* o, const OnDevice& on)
{
    need(PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 3);
    const at::Tensor& turns = on(PyTuple_GET_ITEM(o, 0));
    need(turns.scalar_type() == at::kLong && turns.dim() == 1 && turns.numel() < (1 << 20));
    r->turns = (decltype(r->turns))pointer(turns);
    r->rot_dim = int32_of(2 * turns.numel());
    const int interleaved = PyObject_IsTrue(PyTuple_GET_ITEM(o, 1));
    need(interleaved >= 0);
    r->interleaved = interleaved;
    r->magnitude = float_of(PyTuple_GET_ITEM(o, 2));
}

void fill_paged(fdd_paged_cache* c, PyObject* o, const OnDevice& on)
{
    need(PyTuple_Check(o) && PyTuple_GET_SIZE(o) == 4);
    const at::Tensor &k = on(PyTuple_GET_ITEM(o, 0)), &v = on(PyTuple_GET_ITEM(o, 1)), &table = on(PyTuple_GET_ITEM(o, 2)), &lens = on(PyTuple_GET_ITEM(o, 3));
    need(k.dim() == 4 && v.sizes() == k.sizes() && v.scalar_type() == k.scalar_type());
    need(table.dim() == 2 && table.scalar_type() == at::kInt && lens.dim() == 1 && lens.scalar_type() == at::kInt && lens.size(0) == table.size(0));
    c->k = pointer(k); c->v = pointer(v);
    c->page_table = (const int32_t*)pointer(table); c->lens = (const int32_t*)pointer(lens);
    c->N = int32_of(table.size(0)); c->max_pages = int32_of(table.size(1));
    c->pages = int32_of(k.size(0)); c->Hkv = int32_of(k.size(1)); c->page_size = int32_of(k.size(2)); c->D = int32_of(k.size(3));
    c->dtype = (decltype(c->dtype))dtype_code(k);
}

// q, positions, table, k, out, k_out, inverse, device
void fill_rope(fdd_rope_params* p, PyObject* const* a)
{
    const OnDevice on{int32_of(a[7])};
    const at::Tensor &q = on(a[0]), &pos = on(a[1]), &out = on(a[4]);
    need(q.dim() >= 2);
    const int64_t lead = q.dim() - 2;
    need(pos.scalar_type() == at::kInt && pos.sizes() == q.sizes().slice(0, lead));
    p->rows = int32_of(pos.numel());
    p->Hq = int32_of(q.size(lead)); p->D = int32_of(q.size(lead + 1));
    p->dtype = (decltype(p->dtype))dtype_code(q);
    const int inverse = PyObject_IsTrue(a[6]);
    need(inverse >= 0);
    p->flags = inverse ? FDD_ROPE_INVERSE : 0;
    fill_table(&p->table, a[2], on);
    p->positions = (const int32_t*)pointer(pos);
    need(out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type());
    p->q = even_rows(q, &p->q_stride);
    p->q_out = even_rows(out, &p->q_out_stride);
    if (a[3] == Py_None) {
        need(a[5] == Py_None);
        return;
    }
    const at::Tensor &k = on(a[3]), &k_out = on(a[5]);
    need(k.dim() == q.dim() && k.sizes().slice(0, lead) == q.sizes().slice(0, lead) && k.size(lead + 1) == p->D && k.scalar_type() == q.scalar_type());
    need(k_out.sizes() == k.sizes() && k_out.scalar_type() == k.scalar_type());
    p->Hk = int32_of(k.size(lead));
    p->k = even_rows(k, &p->k_stride);
    p->k_out = even_rows(k_out, &p->k_out_stride);
}

// k, v, cache, table, positions, rows, n_rows, device
void fill_append(AppendCall* c, PyObject* const* a)
{
    const OnDevice on{int32_of(a[7])};
    const at::Tensor &k = on(a[0]), &v = on(a[1]);
    fill_paged(&c->cache, a[2], on);
    need(k.dim() == 4 && v.sizes() == k.sizes() && k.size(0) == c->cache.N && k.size(2) == c->cache.Hkv && k.size(3) == c->cache.D);
    need(dtype_code(k) == c->cache.dtype && v.scalar_type() == k.scalar_type());
    const int64_t N = k.size(0), B = k.size(1);
    c->p.B = int32_of(B);
    c->p.k = even_rows(k, &c->p.k_stride);
    c->p.v = even_rows(v, &c->p.v_stride);
    if (a[3] != Py_None) {
        fill_table(&c->table, a[3], on);
        c->p.rope = &c->table;
    }
    c->p.positions = shaped<const int32_t>(on, a[4], at::kInt, {N, B});
    c->p.rows = shaped<const int32_t>(on, a[5], at::kInt, {N, B});
    c->p.n_rows = shaped<const int32_t>(on, a[6], at::kInt, {N});
}

// parents, lens, n_tokens, mask, positions, device; the request's number is mask's
void fill_tree_mask(fdd_tree_mask_params* p, PyObject* const* a)
{
    const OnDevice on{int32_of(a[5])};
    const at::Tensor& mask = on(a[3]);
    need(mask.dim() == 3);
    const int64_t N = mask.size(0), B = mask.size(1);
    p->N = int32_of(N); p->B = int32_of(B);
    need(a[0] != Py_None && a[4] != Py_None);
    p->parents = per_request<const int32_t>(on, a[0], at::kInt, N, {B}, &p->parents_stride);
    p->lens = shaped<const int32_t>(on, a[1], at::kInt, {N});
    p->n_tokens = shaped<const int32_t>(on, a[2], at::kInt, {N});
    p->mask = shaped<uint64_t>(on, a[3], at::kLong, {N, B, (B + 63) / 64});
    p->positions = shaped<int32_t>(on, a[4], at::kInt, {N, B});
}

// q, cache, block_k, block_v, mask, n_tokens, causal_block, max_len, scale, out, device
void fill_paged_attn(PagedAttnCall* c, PyObject* const* a)
{
    const OnDevice on{int32_of(a[10])};
    const at::Tensor &q = on(a[0]), &k = on(a[2]), &v = on(a[3]), &out = on(a[9]);
    fill_paged(&c->cache, a[1], on);
    fdd_paged_attn_params* const p = &c->p;
    need(q.dim() == 4 && k.dim() == 4 && v.sizes() == k.sizes() && q.size(0) == c->cache.N && q.size(3) == c->cache.D);
    const int64_t N = q.size(0), B = q.size(1);
    need(k.size(0) == N && k.size(1) == B && k.size(2) == c->cache.Hkv && k.size(3) == c->cache.D);
    need(dtype_code(q) == c->cache.dtype && k.scalar_type() == q.scalar_type() && v.scalar_type() == q.scalar_type());
    need(out.sizes() == q.sizes() && out.scalar_type() == q.scalar_type());
    p->B = int32_of(B); p->Hq = int32_of(q.size(2));
    const int causal = PyObject_IsTrue(a[6]);
    need(causal >= 0);
    p->flags = causal ? FDD_ATTN_CAUSAL_BLOCK : 0;
    p->max_len = int32_of(a[7]);
    p->scale = a[8] == Py_None ? 0.f : float_of(a[8]);
    p->q = even_rows(q, &p->q_stride);
    p->block_k = even_rows(k, &p->k_stride);
    p->block_v = even_rows(v, &p->v_stride);
    p->mask = per_request<const uint64_t>(on, a[4], at::kLong, N, {B, (B + 63) / 64}, &p->mask_stride);
    p->n_tokens = shaped<const int32_t>(on, a[5], at::kInt, {N});
    p->out = pointer(out);
}

// logits, tokens, uniforms, parents, draft_logits, n_tokens, temperature, draft_temperature, path, n_path, emitted, chances, device
void fill_tree_verify(fdd_tree_verify_params* p, PyObject* const* a)
{
    const OnDevice on{int32_of(a[12])};
    const at::Tensor& x = on(a[0]);
    need(x.dim() == 3);
    const int64_t N = x.size(0), B = x.size(1);
    p->N = int32_of(N); p->B = int32_of(B); p->V = x.size(2);
    p->dtype = (decltype(p->dtype))dtype_code(x);
    p->temperature = float_of(a[6]);
    p->draft_temperature = float_of(a[7]);
    p->logits = pointer(x);
    p->draft_logits = shaped<const void>(on, a[4], x.scalar_type(), x.sizes());
    need(a[1] != Py_None && a[8] != Py_None && a[9] != Py_None && a[10] != Py_None && a[11] != Py_None);
    p->tokens = shaped<const int32_t>(on, a[1], at::kInt, {N, B});
    p->uniforms = shaped<const float>(on, a[2], at::kFloat, {N, B, 2});
    p->parents = per_request<const int32_t>(on, a[3], at::kInt, N, {B}, &p->parents_stride);
    p->n_tokens = shaped<const int32_t>(on, a[5], at::kInt, {N});
    p->path = shaped<int32_t>(on, a[8], at::kInt, {N, B});
    p->n_path = shaped<int32_t>(on, a[9], at::kInt, {N});
    p->emitted = shaped<int32_t>(on, a[10], at::kInt, {N, B});
    p->chances = shaped<float>(on, a[11], at::kFloat, {N, B});
}

// address of a zeroed struct, then the arguments
template <typename P, int ARGS, void (*FILL)(P*, PyObject* const*)>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (n != ARGS + 1) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    void* p = PyLong_AsVoidPtr(args[0]);
    if (!p) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no address");
        return nullptr;
    }
    bool ok = !at::impl::torch_function_mode_enabled();
    if (ok) {
        try {
            FILL(static_cast<P*>(p), args + 1);
        } catch (...) {       // (NotOrdinary, or an exception of torch's own)
            ok = false;
            PyErr_Clear();
        }
    }
    return PyBool_FromLong(ok);
}

// src, N, dst of a fork into a tensor of the caller's: (bytes, address of src, address of dst), or None
PyObject* fork(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    if (n != 3) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    if (!at::impl::torch_function_mode_enabled()) {
        try {
            const at::Tensor &src = tensor(args[0]), &dst = tensor(args[2]);
            const int64_t N = int32_of(args[1]);
            need(N > 0 && dst.numel() % N == 0 && dst.numel() / N * (int64_t)dst.element_size() == src.numel() * (int64_t)src.element_size());
            void *const from = pointer(src), *const to = pointer(dst);
            return Py_BuildValue("(nKK)", (Py_ssize_t)(src.numel() * src.element_size()), (unsigned long long)reinterpret_cast<uintptr_t>(from),
                                 (unsigned long long)reinterpret_cast<uintptr_t>(to));
        } catch (...) {       // (NotOrdinary, or an exception of torch's own)
            PyErr_Clear();
        }
    }
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"fork", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&fork)), METH_FASTCALL, "arguments of fdd_fork_block"},
    {"attn", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&call<fdd_attn_params, 15, fill_attn>)), METH_FASTCALL, "fill an fdd_attn_params"},
    {"unmask", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&call<fdd_unmask_params, 9, fill_unmask>)), METH_FASTCALL, "fill an fdd_unmask_params"},
    {"quant", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&call<QuantCall, 5, fill_quant>)), METH_FASTCALL, "fill an fdd_quant_cache and the fdd_quant_rows behind it"},
    {"attn_quant", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&call<AttnQuantCall, 15, fill_attn_quant>)), METH_FASTCALL, "fill an fdd_attn_params and the fdd_quant_cache behind it"},
    {"logprobs", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&call<fdd_logprob_params, 10, fill_logprobs>)), METH_FASTCALL, "fill an fdd_logprob_params"},
    {"rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&call<fdd_rope_params, 8, fill_rope>)), METH_FASTCALL, "fill an fdd_rope_params"},
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&call<AppendCall, 8, fill_append>)), METH_FASTCALL, "fill an fdd_paged_cache, the fdd_paged_append_params behind it and their table"},
    {"tree_mask", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&call<fdd_tree_mask_params, 6, fill_tree_mask>)), METH_FASTCALL, "fill an fdd_tree_mask_params"},
    {"paged_attn", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&call<PagedAttnCall, 11, fill_paged_attn>)), METH_FASTCALL, "fill an fdd_paged_cache and the fdd_paged_attn_params behind it"},
    {"tree_verify", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(&call<fdd_tree_verify_params, 13, fill_tree_verify>)), METH_FASTCALL, "fill an fdd_tree_verify_params"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal()
{
    PyObject* m = PyModule_Create(&module);
    if (m && (PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) < 0 ||
              PyModule_AddIntConstant(m, "attn_bytes", sizeof(fdd_attn_params)) < 0 ||
              PyModule_AddIntConstant(m, "unmask_bytes", sizeof(fdd_unmask_params)) < 0 ||
              PyModule_AddIntConstant(m, "quant_bytes", sizeof(QuantCall)) < 0 ||
              PyModule_AddIntConstant(m, "attn_quant_bytes", sizeof(AttnQuantCall)) < 0 ||
              PyModule_AddIntConstant(m, "logprobs_bytes", sizeof(fdd_logprob_params)) < 0 ||
              PyModule_AddIntConstant(m, "rope_bytes", sizeof(fdd_rope_params)) < 0 ||
              PyModule_AddIntConstant(m, "append_bytes", sizeof(AppendCall)) < 0 ||
              PyModule_AddIntConstant(m, "tree_mask_bytes", sizeof(fdd_tree_mask_params)) < 0 ||
              PyModule_AddIntConstant(m, "paged_attn_bytes", sizeof(PagedAttnCall)) < 0 ||
              PyModule_AddIntConstant(m, "tree_verify_bytes", sizeof(fdd_tree_verify_params)) < 0)) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
