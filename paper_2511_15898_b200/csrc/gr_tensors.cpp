// The binding's short way: the checks and the call of the operators around a decoding step for tensors as they come in a decode
// loop.  From Python they cost the host 10 us a call (24 tensors of a state: 18 more), as long as or longer than the GPU needs; here 1.
// Every function answers None where anything is not as it expects (another device than the current one, a list of different
// layouts, a wrong type ...): the binding's own way then looks closer, and raises or makes the call.
#include <Python.h>
#include <math.h>
#include <string.h>
#include <vector>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/Functions.h>
#include "gr.h"

namespace {

const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }

// a contiguous tensor of this type on this device; where `optional`, None is one without an address
bool is_plain(PyObject* o, at::ScalarType kind, c10::Device dev, bool optional, const at::Tensor** out)
{
    *out = nullptr;
    if (o == Py_None) return optional;
    const at::Tensor* t = tensor(o);
    if (!t || !t->is_cuda() || t->device() != dev || t->scalar_type() != kind || t->layout() != at::kStrided || !t->is_contiguous()) return false;
    *out = t;
    return true;
}
template <class T> T* address(const at::Tensor* t) { return t ? reinterpret_cast<T*>(t->data_ptr()) : nullptr; }

// CUDA tensors in a list that all have the first one's shape, strides, type and device
bool all_alike(PyObject* list, std::vector<void*>& at)
{
    if (!PyList_Check(list) || PyList_GET_SIZE(list) == 0) return false;
    const Py_ssize_t n = PyList_GET_SIZE(list);
    at.resize(n);
    const at::Tensor* first = nullptr;
    for (Py_ssize_t i = 0; i < n; i++) {
        const at::Tensor* t = tensor(PyList_GET_ITEM(list, i));
        if (!t || !t->is_cuda() || t->layout() != at::kStrided) return false;
        if (!first) first = t;
        else if (t->device() != first->device() || t->scalar_type() != first->scalar_type() || t->sizes() != first->sizes() || t->strides() != first->strides()) return false;
        at[i] = t->data_ptr();
    }
    return true;
}

// the pieces of a state in x [groups, beams, ...]: how many, elements from one to the next, elements of one
bool pieces(const at::Tensor& x, long token_dim, long long* parts, long long* step, long long* part)
{
    const long from = token_dim < 0 ? 2 : token_dim;
    *part = 1; *parts = 1; *step = 0;
    for (long d = x.dim() - 1; d >= from; d--) {
        if (x.size(d) > 1 && x.stride(d) != *part) return false;
        *part *= x.size(d);
    }
    for (long d = from - 1; d > 1; d--) {
        if (x.size(d) == 1) continue;
        if (*parts > 1 && x.stride(d) != *step * *parts) return false;
        if (*parts == 1) *step = x.stride(d);
        *parts *= x.size(d);
    }
    return true;
}

// whether `dev` is current; its current stream
bool here(c10::Device dev, void** stream)
{
    if (!dev.has_index() || c10::cuda::current_device() != dev.index()) return false;
    *stream = (void*)c10::cuda::getCurrentCUDAStream(dev.index()).stream();
    return true;
}

#define GR_OR_NONE(condition) do { if (!(condition)) { PyErr_Clear(); Py_RETURN_NONE; } } while (0)
#define GR_TRY try {
#define GR_CATCH } catch (...) { PyErr_Clear(); Py_RETURN_NONE; }

// reorder(function, states, parents, lengths, token_dim, out) -> its answer or None
PyObject* reorder(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    GR_OR_NONE(n == 6);
    GR_TRY
    auto* f = reinterpret_cast<decltype(&gr_reorder_states)>(PyLong_AsVoidPtr(a[0]));
    std::vector<void*> src, dst;
    GR_OR_NONE(f && all_alike(a[1], src));
    const at::Tensor& x = *tensor(PyList_GET_ITEM(a[1], 0));
    const at::Tensor *y = &x, *parents, *lengths;
    const c10::Device dev = x.device();
    const bool in_place = a[5] == Py_None;
    const long token_dim = a[4] == Py_None ? -1 : PyLong_AsLong(a[4]);
    GR_OR_NONE(!PyErr_Occurred() && (a[4] == Py_None || token_dim >= 0));
    GR_OR_NONE(is_plain(a[2], at::kInt, dev, false, &parents) && is_plain(a[3], at::kInt, dev, true, &lengths));
    GR_OR_NONE(x.dim() >= 2 && parents->dim() == 2 && parents->size(0) == x.size(0) && (lengths != nullptr) == (token_dim >= 0));
    GR_OR_NONE(token_dim < 0 || (token_dim >= 2 && token_dim < x.dim()));
    GR_OR_NONE(!lengths || (lengths->dim() == 2 && lengths->size(0) == x.size(0) && lengths->size(1) == x.size(1)));
    const long long chosen = parents->size(1);
    if (!in_place) {
        GR_OR_NONE(all_alike(a[5], dst) && dst.size() == src.size());
        y = tensor(PyList_GET_ITEM(a[5], 0));
        GR_OR_NONE(y->device() == dev && y->scalar_type() == x.scalar_type() && y->dim() == x.dim() && y->size(0) == x.size(0) && y->size(1) == chosen);
        for (long d = 2; d < x.dim(); d++) GR_OR_NONE(y->size(d) == x.size(d));
    }
    long long parts, step, part, parts_y, step_y, part_y;
    GR_OR_NONE(pieces(x, token_dim, &parts, &step, &part) && pieces(*y, token_dim, &parts_y, &step_y, &part_y));
    GR_OR_NONE(x.size(0) > 0 && x.size(1) > 0 && chosen > 0 && part > 0 && parts > 0 && parts < (1ll << 31) && x.size(0) < (1ll << 31) && x.size(1) <= GR_MAX_BEAMS && chosen <= GR_MAX_BEAMS);
    const long long e = x.element_size();
    gr_state_layout L;
    L.batch = (int)x.size(0); L.beams_in = (int)x.size(1); L.beams_out = (int)chosen; L.parts = (int)parts;
    L.src_group = x.size(0) > 1 ? x.stride(0) * e : 0; L.src_beam = x.size(1) > 1 ? x.stride(1) * e : 0; L.src_part = step * e;
    L.dst_group = y->size(0) > 1 ? y->stride(0) * e : 0; L.dst_beam = y->size(1) > 1 ? y->stride(1) * e : 0; L.dst_part = step_y * e;
    L.part_bytes = part * e;
    L.token_bytes = token_dim < 0 ? e : part / x.size(token_dim) * e;
    void* stream;
    GR_OR_NONE(here(dev, &stream));
    return PyLong_FromLong(f(src.data(), in_place ? src.data() : dst.data(), (int)src.size(), &L, address<int>(parents), address<int>(lengths), stream));
    GR_CATCH
}

// copy(function, caches, copy_src, copy_dst) -> its answer or None
PyObject* copy(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    GR_OR_NONE(n == 4);
    GR_TRY
    auto* f = reinterpret_cast<decltype(&gr_copy_blocks)>(PyLong_AsVoidPtr(a[0]));
    std::vector<void*> at;
    GR_OR_NONE(f && all_alike(a[1], at));
    const at::Tensor& x = *tensor(PyList_GET_ITEM(a[1], 0));
    const at::Tensor *src, *dst;
    GR_OR_NONE(is_plain(a[2], at::kInt, x.device(), false, &src) && is_plain(a[3], at::kInt, x.device(), false, &dst));
    GR_OR_NONE(x.dim() >= 1 && src->dim() == 1 && dst->dim() == 1 && src->size(0) == dst->size(0) && src->size(0) < (1ll << 31));
    long long per = 1;
    for (long d = x.dim() - 1; d >= 1; d--) {
        GR_OR_NONE(x.size(d) == 1 || x.stride(d) == per);
        per *= x.size(d);
    }
    GR_OR_NONE(x.size(0) > 0 && x.size(0) < (1ll << 31) && per > 0 && (x.size(0) == 1 || x.stride(0) >= per));
    const long long e = x.element_size();
    void* stream;
    GR_OR_NONE(here(x.device(), &stream));
    return PyLong_FromLong(f(at.data(), (int)at.size(), (int)x.size(0), (x.size(0) > 1 ? x.stride(0) : per) * e, per * e, address<int>(src),
                             address<int>(dst), (int)src->size(0), stream));
    GR_CATCH
}

// plan(function, table, lengths, refs, block_size, beams, append, max_tokens, keep, parents, workspace, slots, positions, offsets,
// copy_src, copy_dst, status) -> its answer or None.  (The last seven are the binding's own, made for the shape.)
PyObject* plan(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    GR_OR_NONE(n == 17);
    GR_TRY
    auto* f = reinterpret_cast<decltype(&gr_block_plan)>(PyLong_AsVoidPtr(a[0]));
    const at::Tensor* table = tensor(a[1]);
    GR_OR_NONE(f && table && table->dim() == 2);
    const c10::Device dev = table->device();
    const at::Tensor *lengths, *refs, *append, *keep, *parents, *own[7];
    GR_OR_NONE(is_plain(a[1], at::kInt, dev, false, &table) && is_plain(a[2], at::kInt, dev, false, &lengths) && is_plain(a[3], at::kInt, dev, false, &refs)
               && is_plain(a[6], at::kInt, dev, false, &append) && is_plain(a[8], at::kInt, dev, true, &keep) && is_plain(a[9], at::kInt, dev, true, &parents));
    const long long rows = table->size(0);
    const long block = PyLong_AsLong(a[4]), beams = PyLong_AsLong(a[5]), tokens = PyLong_AsLong(a[7]);
    GR_OR_NONE(rows > 0 && rows < (1ll << 31) && table->size(1) < (1ll << 31) && refs->dim() == 1 && refs->size(0) < (1ll << 31));
    GR_OR_NONE(block > 0 && block < (1l << 31) && beams > 0 && beams <= GR_MAX_BEAMS && tokens >= 0 && tokens < (1l << 31));
    GR_OR_NONE(lengths->dim() == 1 && lengths->size(0) == rows && append->dim() == 1 && append->size(0) == rows && (!keep || (keep->dim() == 1 && keep->size(0) == rows)));
    GR_OR_NONE(!parents || (parents->dim() == 1 && parents->size(0) == rows) || (parents->dim() == 2 && parents->size(0) * beams == rows && parents->size(1) == beams));
    for (int i = 0; i < 7; i++) GR_OR_NONE((own[i] = tensor(a[10 + i])) && own[i]->device() == dev);
    void* stream;
    GR_OR_NONE(here(dev, &stream));
    return PyLong_FromLong(f(address<int>(table), (int)rows, (int)table->size(1), (int)beams, (int)block, address<int>(lengths), address<int>(refs),
                             (int)refs->size(0), address<int>(parents), address<int>(keep), address<int>(append), (int)tokens, own[0]->data_ptr(),
                             address<long long>(own[1]), address<int>(own[2]), address<int>(own[3]), address<int>(own[4]), address<int>(own[5]),
                             address<int>(own[6]), stream));
    GR_CATCH
}

// select(function, logits, scores, select, temperature, lengths, done, eos, length_penalty, workspace, token, parent, score, length,
// done (out), status) -> its answer or None.  (The last seven are the binding's own, made for the shape.)
PyObject* select_(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    GR_OR_NONE(n == 16);
    GR_TRY
    auto* f = reinterpret_cast<decltype(&gr_beam_select)>(PyLong_AsVoidPtr(a[0]));
    const at::Tensor* x = tensor(a[1]);
    GR_OR_NONE(f && x && x->is_cuda() && x->dim() == 3 && x->layout() == at::kStrided && x->numel() > 0);
    GR_OR_NONE(x->scalar_type() == at::kFloat || x->scalar_type() == at::kBFloat16);
    const c10::Device dev = x->device();
    const at::Tensor *scores, *lengths, *done, *own[7];
    const bool bytes = tensor(a[6]) && tensor(a[6])->scalar_type() == at::kByte;
    GR_OR_NONE(is_plain(a[2], at::kFloat, dev, false, &scores) && is_plain(a[5], at::kInt, dev, true, &lengths) && is_plain(a[6], bytes ? at::kByte : at::kBool, dev, true, &done));
    const long long B = x->size(0), W = x->size(1), V = x->size(2), ld = W > 1 ? x->stride(1) : B > 1 ? x->stride(0) : V;
    GR_OR_NONE((V == 1 || x->stride(2) == 1) && (B == 1 || W == 1 || x->stride(0) == W * ld) && ld >= V && B < (1ll << 31) && W <= GR_MAX_BEAMS && V < (1ll << 31));
    for (const at::Tensor* t : {scores, lengths, done}) GR_OR_NONE(!t || (t->dim() == 2 && t->size(0) == B && t->size(1) == W));
    for (int i = 0; i < 7; i++) GR_OR_NONE((own[i] = tensor(a[9 + i])) && own[i]->device() == dev);
    GR_OR_NONE(scores->data_ptr() != own[3]->data_ptr() && (!lengths || lengths->data_ptr() != own[4]->data_ptr()) && (!done || done->data_ptr() != own[5]->data_ptr()));
    const long K = PyLong_AsLong(a[3]), eos = PyLong_AsLong(a[7]);
    const double temperature = PyFloat_AsDouble(a[4]), penalty = PyFloat_AsDouble(a[8]);
    GR_OR_NONE(!PyErr_Occurred() && K > 0 && K <= GR_MAX_SELECT && eos >= -1 && eos < V);
    void* stream;
    GR_OR_NONE(here(dev, &stream));
    return PyLong_FromLong(f(x->data_ptr(), x->scalar_type() == at::kFloat ? GR_F32 : GR_BF16, (int)V, ld, (int)W, (int)B, (float)temperature,
                             address<float>(scores), address<int>(lengths), address<unsigned char>(done), (int)eos, (float)penalty, (int)K, own[0]->data_ptr(),
                             address<int>(own[1]), address<int>(own[2]), address<float>(own[3]), lengths ? address<int>(own[4]) : nullptr,
                             address<unsigned char>(own[5]), address<int>(own[6]), stream));
    GR_CATCH
}

// ---------------------------------------------------------------- paged caches

int type_code(at::ScalarType t) { return t == at::kFloat ? GR_F32 : t == at::kBFloat16 ? GR_BF16 : t == at::kHalf ? GR_F16 : -1; }

// the layout of a cache (keys, values, block_size, heads, dim); its keys
const at::Tensor* cache_of(PyObject* const* a, gr_cache_layout* L, void** values)
{
    const at::Tensor* k = tensor(a[0]);
    if (!k || !k->is_cuda() || k->layout() != at::kStrided || k->dim() != 4 || k->numel() == 0) return nullptr;
    const long block = PyLong_AsLong(a[2]), heads = PyLong_AsLong(a[3]), dim = PyLong_AsLong(a[4]);
    if (PyErr_Occurred() || block < 1 || block >= (1l << 31) || heads < 1 || heads > GR_MAX_HEADS || dim < 1 || dim > GR_MAX_DIM || k->size(0) >= (1ll << 31)) return nullptr;
    L->heads = (int)heads; L->dim = (int)dim; L->block_size = (int)block; L->num_blocks = (int)k->size(0);
    L->token_stride = L->head_stride = 0;
    *values = nullptr;
    if (k->scalar_type() == at::kByte) {
        if (a[1] != Py_None || block % 8 || dim % 32 || k->size(1) != heads || k->size(2) != block / 8 || k->size(3) != 9 * dim) return nullptr;
        long long per = 1;
        for (long d = 3; d >= 1; d--) { if (k->size(d) > 1 && k->stride(d) != per) return nullptr; per *= k->size(d); }
        L->format = GR_Q4; L->block_stride = k->size(0) > 1 ? k->stride(0) : per;
        return k;
    }
    const at::Tensor* v = tensor(a[1]);
    L->format = type_code(k->scalar_type());
    if (L->format < 0 || !v || v->device() != k->device() || v->scalar_type() != k->scalar_type() || v->sizes() != k->sizes() || v->strides() != k->strides()) return nullptr;
    if (k->size(1) != block || k->size(2) != heads || k->size(3) != dim || (dim > 1 && k->stride(3) != 1)) return nullptr;
    L->block_stride = k->stride(0); L->token_stride = k->stride(1); L->head_stride = k->stride(2);
    *values = v->data_ptr();
    return k;
}
// a [tokens, heads, dim] tensor of this type and device whose heads' elements lie next to one another
const at::Tensor* rows_of(PyObject* o, at::ScalarType kind, c10::Device dev, long long tokens, long long heads, long long dim)
{
    const at::Tensor* t = tensor(o);
    return t && t->is_cuda() && t->layout() == at::kStrided && t->device() == dev && t->scalar_type() == kind && t->dim() == 3 && t->size(0) == tokens
           && t->size(1) == heads && t->size(2) == dim && (dim == 1 || t->stride(2) == 1) ? t : nullptr;
}

// append(function, keys, values, block_size, heads, dim, k, v, slots, positions, frequencies, interleaved, q, q_out) -> its answer or None
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    GR_OR_NONE(n == 14);
    GR_TRY
    auto* f = reinterpret_cast<decltype(&gr_cache_append)>(PyLong_AsVoidPtr(a[0]));
    gr_cache_layout L;
    void* values;
    const at::Tensor *keys = cache_of(a + 1, &L, &values), *k = tensor(a[6]), *slots, *positions, *freq;
    GR_OR_NONE(f && keys && k && k->dim() == 3 && type_code(k->scalar_type()) >= 0 && k->size(0) < (1ll << 31));
    const c10::Device dev = keys->device();
    const long long T = k->size(0);
    const at::Tensor* v = rows_of(a[7], k->scalar_type(), dev, T, L.heads, L.dim);
    GR_OR_NONE(v && rows_of(a[6], k->scalar_type(), dev, T, L.heads, L.dim));
    GR_OR_NONE(is_plain(a[8], at::kLong, dev, false, &slots) && is_plain(a[9], at::kInt, dev, true, &positions) && is_plain(a[10], at::kDouble, dev, true, &freq));
    GR_OR_NONE(slots->dim() == 1 && slots->size(0) == T && (!positions || (positions->dim() == 1 && positions->size(0) == T)));
    GR_OR_NONE(!freq || (positions && freq->dim() == 1 && 2 * freq->size(0) <= L.dim));
    gr_cache_tokens X = {};
    X.k = k->data_ptr(); X.v = v->data_ptr(); X.dtype = type_code(k->scalar_type());
    X.k_token = k->stride(0); X.k_head = k->stride(1); X.v_token = v->stride(0); X.v_head = v->stride(1);
    if (a[12] != Py_None) {
        const at::Tensor* q = tensor(a[12]);
        GR_OR_NONE(q && q->dim() == 3 && q->size(1) <= GR_MAX_HEADS);
        const at::Tensor* out = rows_of(a[13], k->scalar_type(), dev, T, q->size(1), L.dim);
        GR_OR_NONE(out && rows_of(a[12], k->scalar_type(), dev, T, q->size(1), L.dim));
        X.q = q->data_ptr(); X.q_out = out->data_ptr(); X.q_heads = (int)q->size(1);
        X.q_token = q->stride(0); X.q_head = q->stride(1); X.out_token = out->stride(0); X.out_head = out->stride(1);
    } else GR_OR_NONE(a[13] == Py_None);
    const int interleaved = PyObject_IsTrue(a[11]);
    void* stream;
    GR_OR_NONE(interleaved >= 0 && here(dev, &stream));
    return PyLong_FromLong(f(keys->data_ptr(), values, &L, &X, (int)T, address<long long>(slots), address<int>(positions), address<double>(freq),
                             freq ? 2 * (int)freq->size(0) : 0, interleaved, stream));
    GR_CATCH
}

// read(function, keys, values, block_size, heads, dim, slots, dtype, k, v) -> (k, v), its answer where that is not 0, or None.  Without k and v: new ones of
// type dtype.
PyObject* read(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    GR_OR_NONE(n == 10);
    GR_TRY
    auto* f = reinterpret_cast<decltype(&gr_cache_read)>(PyLong_AsVoidPtr(a[0]));
    gr_cache_layout L;
    void* values;
    const at::Tensor *keys = cache_of(a + 1, &L, &values), *slots;
    GR_OR_NONE(f && keys && is_plain(a[6], at::kLong, keys->device(), false, &slots) && slots->dim() == 1 && slots->size(0) < (1ll << 31));
    const c10::Device dev = keys->device();
    const long long T = slots->size(0);
    void* stream;
    GR_OR_NONE(here(dev, &stream));
    at::Tensor k, v;
    if (a[8] == Py_None) {
        GR_OR_NONE(a[9] == Py_None && THPDtype_Check(a[7]));
        const at::ScalarType kind = reinterpret_cast<THPDtype*>(a[7])->scalar_type;
        GR_OR_NONE(type_code(kind) >= 0);
        const auto as = at::TensorOptions().dtype(kind).device(dev);
        k = at::empty({T, L.heads, L.dim}, as);
        v = at::empty({T, L.heads, L.dim}, as);
    } else {
        const at::Tensor* out = tensor(a[8]);
        GR_OR_NONE(out && type_code(out->scalar_type()) >= 0);
        const at::Tensor *x = rows_of(a[8], out->scalar_type(), dev, T, L.heads, L.dim), *y = rows_of(a[9], out->scalar_type(), dev, T, L.heads, L.dim);
        GR_OR_NONE(x && y);
        k = *x; v = *y;
    }
    const int rc = f(keys->data_ptr(), values, &L, address<long long>(slots), (int)T, type_code(k.scalar_type()), k.data_ptr(), k.stride(0), k.stride(1),
                     v.data_ptr(), v.stride(0), v.stride(1), stream);
    if (rc != GR_OK) return PyLong_FromLong(rc);
    PyObject *x = THPVariable_Wrap(k), *y = THPVariable_Wrap(v), *both = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x); Py_XDECREF(y);
    return both;
    GR_CATCH
}

// attend(function, q, keys, values, block_size, heads, dim, table, offsets, positions, scale, window, workspace, out, status, workspace's size) -> its answer
// or None.
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    GR_OR_NONE(n == 16);
    GR_TRY
    auto* f = reinterpret_cast<decltype(&gr_cache_attend)>(PyLong_AsVoidPtr(a[0]));
    auto* bytes = reinterpret_cast<decltype(&gr_attend_workspace_bytes)>(PyLong_AsVoidPtr(a[15]));
    gr_cache_layout L;
    void* values;
    const at::Tensor *q = tensor(a[1]), *keys = cache_of(a + 2, &L, &values), *table, *offsets, *positions;
    GR_OR_NONE(f && bytes && q && keys && L.format == GR_Q4 && q->dim() == 3 && (q->scalar_type() == at::kBFloat16 || q->scalar_type() == at::kHalf));
    const c10::Device dev = keys->device();
    const long long T = q->size(0), heads = q->size(1);
    GR_OR_NONE(T < (1ll << 31) && heads <= GR_MAX_HEADS && rows_of(a[1], q->scalar_type(), dev, T, heads, L.dim));
    GR_OR_NONE(is_plain(a[7], at::kInt, dev, false, &table) && is_plain(a[8], at::kInt, dev, false, &offsets) && is_plain(a[9], at::kInt, dev, false, &positions));
    GR_OR_NONE(table->dim() == 2 && table->size(0) < (1ll << 31) - 1 && table->size(1) < (1ll << 31) && offsets->dim() == 1 && offsets->size(0) == table->size(0) + 1
               && positions->dim() == 1 && positions->size(0) == T);
    const at::Tensor *workspace = tensor(a[12]), *out = rows_of(a[13], q->scalar_type(), dev, T, heads, L.dim), *status = tensor(a[14]);
    GR_OR_NONE(workspace && out && workspace->device() == dev && workspace->scalar_type() == at::kByte && workspace->is_contiguous());
    const size_t least = bytes(L.heads, (int)heads, L.dim, (int)table->size(0), (int)T);
    GR_OR_NONE(least > 0 && (size_t)workspace->numel() >= least && is_plain(a[14], at::kInt, dev, false, &status) && status->numel() == table->size(0));
    const double scale = a[10] == Py_None ? pow((double)L.dim, -0.5) : PyFloat_AsDouble(a[10]);
    const long window = PyLong_AsLong(a[11]);
    GR_OR_NONE(!PyErr_Occurred() && window >= 0 && window < (1l << 31));
    void* stream;
    GR_OR_NONE(here(dev, &stream));
    return PyLong_FromLong(f(q->data_ptr(), type_code(q->scalar_type()), (int)heads, q->stride(0), q->stride(1), keys->data_ptr(), &L, address<int>(table),
                             (int)table->size(1), (int)table->size(0), address<int>(offsets), address<int>(positions), (int)T, (float)scale, (int)window,
                             workspace->data_ptr(), out->data_ptr(), out->stride(0), out->stride(1), address<int>(status), stream));
    GR_CATCH
}

// logprobs(function, logits, tokens, top, temperature, logprob, entropy, top_token, top_logprob, status) -> its answer or None.
PyObject* logprobs(PyObject*, PyObject* const* a, Py_ssize_t n)
{
    GR_OR_NONE(n == 10);
    GR_TRY
    auto* f = reinterpret_cast<decltype(&gr_token_logprobs)>(PyLong_AsVoidPtr(a[0]));
    const at::Tensor *x = tensor(a[1]), *tokens, *own[5];
    GR_OR_NONE(f && x && x->is_cuda() && x->dim() == 2 && x->layout() == at::kStrided && x->numel() > 0);
    GR_OR_NONE(x->scalar_type() == at::kFloat || x->scalar_type() == at::kBFloat16);
    const c10::Device dev = x->device();
    const long long R = x->size(0), V = x->size(1), ld = R > 1 ? x->stride(0) : V;
    GR_OR_NONE((V == 1 || x->stride(1) == 1) && ld >= V && R < (1ll << 31) && V < (1ll << 31));
    GR_OR_NONE(is_plain(a[2], at::kInt, dev, true, &tokens) && (!tokens || ((tokens->dim() == 1 || tokens->dim() == 2) && tokens->size(0) == R)));
    const long long given = !tokens ? 0 : tokens->dim() == 1 ? 1 : tokens->size(1);
    const long top = PyLong_AsLong(a[3]);
    const double temperature = PyFloat_AsDouble(a[4]);
    GR_OR_NONE(!PyErr_Occurred() && top >= 0 && top <= GR_MAX_SELECT && given <= GR_MAX_GIVEN);
    for (int i = 0; i < 5; i++) GR_OR_NONE(is_plain(a[5 + i], i == 2 || i == 4 ? at::kInt : at::kFloat, dev, false, &own[i]));
    GR_OR_NONE(own[0]->numel() == R * given && own[1]->numel() == R && own[2]->numel() == R * top && own[3]->numel() == R * top && own[4]->numel() == R);
    GR_OR_NONE(!tokens || top == 0 || tokens->data_ptr() != own[2]->data_ptr());
    void* stream;
    GR_OR_NONE(here(dev, &stream));
    return PyLong_FromLong(f(x->data_ptr(), x->scalar_type() == at::kFloat ? GR_F32 : GR_BF16, (int)V, ld, (int)R, (float)temperature, address<int>(tokens),
                             (int)given, (int)top, address<float>(own[0]), address<float>(own[1]), address<int>(own[2]), address<float>(own[3]),
                             address<int>(own[4]), stream));
    GR_CATCH
}

PyMethodDef methods[] = {{"reorder", (PyCFunction)(void (*)(void))reorder, METH_FASTCALL, nullptr}, {"copy", (PyCFunction)(void (*)(void))copy, METH_FASTCALL, nullptr},
                         {"plan", (PyCFunction)(void (*)(void))plan, METH_FASTCALL, nullptr}, {"select", (PyCFunction)(void (*)(void))select_, METH_FASTCALL, nullptr},
                         {"append", (PyCFunction)(void (*)(void))append, METH_FASTCALL, nullptr}, {"read", (PyCFunction)(void (*)(void))read, METH_FASTCALL, nullptr},
                         {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, nullptr}, {"logprobs", (PyCFunction)(void (*)(void))logprobs, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// (torch's objects are looked into directly: with another torch than the one it was compiled for the binding leaves it alone)
PyMODINIT_FUNC PyInit__tensors(void)
{
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", GR_TORCH_VERSION) != 0) Py_CLEAR(m);
    return m;
}
