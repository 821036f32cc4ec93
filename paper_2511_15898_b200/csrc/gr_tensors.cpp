// The binding's short way: the checks and the call of the operators around a decoding step for tensors as they come in a decode
// loop.  From Python they cost the host 10 us a call (24 tensors of a state: 18 more), as long as or longer than the GPU needs; here 1.
// Every function answers None where anything is not as it expects (another device than the current one, a list of different
// layouts, a wrong type ...): the binding's own way then looks closer, and raises or makes the call.
#include <Python.h>
#include <string.h>
#include <vector>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>
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

PyMethodDef methods[] = {{"reorder", (PyCFunction)(void (*)(void))reorder, METH_FASTCALL, nullptr}, {"copy", (PyCFunction)(void (*)(void))copy, METH_FASTCALL, nullptr},
                         {"plan", (PyCFunction)(void (*)(void))plan, METH_FASTCALL, nullptr}, {"select", (PyCFunction)(void (*)(void))select_, METH_FASTCALL, nullptr},
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
