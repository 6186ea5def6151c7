// binding.cpp -- the calls of a decode step with drafted tokens, from Python objects straight
// to the library.  Each function looks at its tensors, allocates what is not given and
// enqueues, in some three microseconds where the same in Python takes fifteen: what these
// calls cost is the host's.  Where anything is not as it should be, or is not plain (another
// device than the current one, tensors that require gradients, sizes to be read from the device),
// it does nothing and returns None, and ops.py goes the whole way, which says what is wrong.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "e2ops.h"

namespace {

// A tensor of a call, on its device, without a gradient to keep; null: not so.
struct Call {
    int device;
    bool grad, ok = true;

    explicit Call(int device) : device(device), grad(c10::GradMode::is_enabled()) { ok = c10::cuda::current_device() == device; }

    const at::Tensor *tensor(PyObject *o, c10::ScalarType type, int64_t dims)
    {
        if (ok && THPVariable_CheckExact(o)) {
            const at::Tensor &t = THPVariable_Unpack(o);
            if (t.is_cuda() && t.get_device() == device && t.scalar_type() == type && t.dim() == dims && t.layout() == c10::kStrided &&
                !(grad && t.requires_grad()))
                return &t;
        }
        ok = false;
        return nullptr;
    }
    // [n], side by side
    const at::Tensor *vector(PyObject *o, c10::ScalarType type, int64_t n)
    {
        const at::Tensor *t = tensor(o, type, 1);
        if (t && (t->size(0) != n || t->stride(0) != 1)) ok = false;
        return ok ? t : nullptr;
    }
    // [rows][cols], rows side by side in themselves
    const at::Tensor *matrix(PyObject *o, c10::ScalarType type)
    {
        const at::Tensor *t = tensor(o, type, 2);
        if (t && (t->size(0) < 1 || t->size(1) < 1 || (t->size(1) > 1 && t->stride(1) != 1) || !fits(t->size(0)) || !fits(t->size(1)))) ok = false;
        return ok ? t : nullptr;
    }
    // [tokens][heads][dim], a token's heads side by side
    const at::Tensor *heads(PyObject *o, c10::ScalarType type, int64_t dim)
    {
        const at::Tensor *t = tensor(o, type, 3);
        if (t && (t->size(0) < 1 || t->size(1) < 1 || t->size(2) != dim || t->stride(2) != 1 || (t->size(1) > 1 && t->stride(1) != dim) ||
                  !fits(t->size(0)) || !fits(t->size(1))))
            ok = false;
        return ok ? t : nullptr;
    }
    int64_t integer(PyObject *o, int64_t least, int64_t most)
    {
        int overflow = 0;
        const int64_t x = PyLong_CheckExact(o) ? PyLong_AsLongLongAndOverflow(o, &overflow) : least - 1;
        if (overflow || x < least || x > most) ok = false;
        return x;
    }
    static bool fits(int64_t n) { return n <= 0x7fffffff; }
    static int64_t stride(const at::Tensor &t, int64_t row) { return t.size(0) > 1 ? t.stride(0) : row; }
    void *stream() const { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }
    at::Tensor empty(at::IntArrayRef shape, c10::ScalarType type) const
    {
        return at::empty(shape, at::TensorOptions().dtype(type).device(c10::Device(c10::kCUDA, (c10::DeviceIndex)device)));
    }
};

int type_of(c10::ScalarType t) { return t == c10::kHalf ? E2_F16 : t == c10::kBFloat16 ? E2_BF16 : t == c10::kFloat ? E2_F32 : -1; }
c10::ScalarType type_of(PyObject *o) { return THPVariable_CheckExact(o) ? THPVariable_Unpack(o).scalar_type() : c10::kByte; }
template <class T> const T *data(const at::Tensor *t) { return t ? static_cast<const T *>(t->const_data_ptr()) : nullptr; }

// (address of the struct, device, whether it requires gradients)
template <class T> const T *handle(PyObject *o, int &device, bool &grad)
{
    device = (int)PyLong_AsLong(PyTuple_GET_ITEM(o, 1));
    grad = PyTuple_GET_ITEM(o, 2) == Py_True;
    return static_cast<const T *>(PyLong_AsVoidPtr(PyTuple_GET_ITEM(o, 0)));
}

// cache, q, parents, table, lens, starts, max_new, max_len, scale, window, out, workspace
PyObject *attend_tree(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 12) Py_RETURN_NONE;
    int device;
    bool grad;
    const e2_cache *c = handle<e2_cache>(a[0], device, grad);
    Call call(device);
    if (grad && call.grad) Py_RETURN_NONE;
    const c10::ScalarType type = type_of(a[1]);
    if (type != c10::kHalf && type != c10::kBFloat16) Py_RETURN_NONE;
    const at::Tensor *q = call.heads(a[1], type, c->head_dim), *table = call.matrix(a[3], c10::kInt);
    if (!call.ok) Py_RETURN_NONE;
    const int64_t tokens = q->size(0), heads = q->size(1), batch = table->size(0), row = heads * c->head_dim;
    const at::Tensor *parents = call.vector(a[2], c10::kInt, tokens), *lens = call.vector(a[4], c10::kInt, batch),
                     *starts = call.vector(a[5], c10::kInt, batch + 1);
    e2_attend_args args{};
    args.max_new = (int32_t)call.integer(a[6], 0, 0x7fffffff);
    args.max_len = (int32_t)call.integer(a[7], 0, 0x7fffffff);
    args.window = (int32_t)call.integer(a[9], 0, 0x7fffffff);
    args.scale = c->head_dim == 64 ? 0.125f : 0.08838834764831845f;
    if (a[8] != Py_None) {
        if (!PyFloat_CheckExact(a[8])) Py_RETURN_NONE;
        args.scale = (float)PyFloat_AS_DOUBLE(a[8]);
    }
    at::Tensor out;
    if (a[10] != Py_None) {
        const at::Tensor *given = call.heads(a[10], type, c->head_dim);
        if (!call.ok || given->size(0) != tokens || given->size(1) != heads) Py_RETURN_NONE;
        out = *given;
    }
    if (!call.ok || (a[11] != Py_None && !THPVariable_CheckExact(a[11]))) Py_RETURN_NONE;
    try {
        if (!out.defined()) out = call.empty({tokens, heads, c->head_dim}, type);
        args.tokens = (int32_t)tokens, args.dtype = type_of(type), args.q_heads = (int32_t)heads, args.batch = (int32_t)batch;
        args.table = data<int32_t>(table), args.table_cols = (int32_t)table->size(1), args.table_stride = Call::stride(*table, table->size(1));
        args.lens = data<int32_t>(lens), args.starts = data<int32_t>(starts);
        args.q = data<void>(q), args.q_stride = Call::stride(*q, row);
        args.out = out.data_ptr(), args.out_stride = Call::stride(out, row);
        at::Tensor workspace;
        if (a[11] != Py_None) {
            workspace = THPVariable_Unpack(a[11]);
            if (!workspace.is_cuda() || !workspace.is_contiguous()) Py_RETURN_NONE;
        } else if (const size_t need = e2_cache_attend_tree_workspace(c, &args)) {
            workspace = call.empty({(int64_t)need}, c10::kByte);
        }
        if (e2_cache_attend_tree(c, &args, data<int32_t>(parents), workspace.defined() ? workspace.data_ptr() : nullptr,
                                 workspace.defined() ? workspace.nbytes() : 0, call.stream()) != E2_OK)
            Py_RETURN_NONE;
    } catch (...) {
        Py_RETURN_NONE;                      // (no memory, say: Python's way meets it again)
    }
    return THPVariable_Wrap(std::move(out));
}

// device, logits, ids, parents, starts, uniforms, draft, temperature, max_new
PyObject *verify(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 8 || !THPVariable_CheckExact(a[0])) Py_RETURN_NONE;
    const c10::ScalarType type = type_of(a[0]);
    if (type_of(type) < 0 || !THPVariable_Unpack(a[0]).is_cuda() || !THPVariable_CheckExact(a[3]) || THPVariable_Unpack(a[3]).dim() != 1) Py_RETURN_NONE;
    Call call(THPVariable_Unpack(a[0]).get_device());
    const at::Tensor *logits = call.matrix(a[0], type);
    if (!call.ok) Py_RETURN_NONE;
    const int64_t tokens = logits->size(0), vocab = logits->size(1), batch = THPVariable_Unpack(a[3]).size(0) - 1;
    const at::Tensor *ids = call.vector(a[1], c10::kInt, tokens), *parents = call.vector(a[2], c10::kInt, tokens),
                     *starts = call.vector(a[3], c10::kInt, batch + 1), *uniforms = call.vector(a[4], c10::kFloat, tokens), *draft = nullptr,
                     *temperature = nullptr;
    if (a[5] != Py_None) draft = call.matrix(a[5], type);
    if (a[6] != Py_None) temperature = call.vector(a[6], c10::kFloat, batch);
    const int64_t most = call.integer(a[7], 0, E2_MAX_DRAFT);
    if (!call.ok || batch < 1 || (draft && (draft->size(0) != tokens || draft->size(1) != vocab))) Py_RETURN_NONE;
    PyObject *result = nullptr;
    try {
        at::Tensor kept = call.empty({batch}, c10::kInt), nodes = call.empty({batch, most}, c10::kInt), answer = call.empty({batch, most}, c10::kInt);
        e2_verify_args args{};
        args.tokens = (int32_t)tokens, args.vocab = (int32_t)vocab, args.dtype = type_of(type), args.batch = (int32_t)batch;
        args.max_new = (int32_t)most;
        args.logits = data<void>(logits), args.logits_stride = Call::stride(*logits, vocab);
        args.draft = data<void>(draft), args.draft_stride = draft ? Call::stride(*draft, vocab) : 0;
        args.ids = data<int32_t>(ids), args.parents = data<int32_t>(parents), args.starts = data<int32_t>(starts);
        args.uniforms = data<float>(uniforms), args.temperature = data<float>(temperature);
        args.kept = kept.data_ptr<int32_t>(), args.nodes = nodes.data_ptr<int32_t>(), args.answer = answer.data_ptr<int32_t>();
        if (e2_verify_drafts(&args, call.stream()) != E2_OK) Py_RETURN_NONE;
        result = PyTuple_New(3);
        if (!result) return nullptr;
        PyTuple_SET_ITEM(result, 0, THPVariable_Wrap(std::move(kept)));
        PyTuple_SET_ITEM(result, 1, THPVariable_Wrap(std::move(nodes)));
        PyTuple_SET_ITEM(result, 2, THPVariable_Wrap(std::move(answer)));
    } catch (...) {
        Py_XDECREF(result);
        Py_RETURN_NONE;
    }
    return result;
}

// layers (and their number, and the address of their arrays), table, lens, starts, nodes, kept, lens_out
PyObject *keep(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    if (n != 7) Py_RETURN_NONE;
    int device;
    bool grad;
    const e2_cache *c = handle<e2_cache>(a[0], device, grad);
    Call call(device);
    if (grad && call.grad) Py_RETURN_NONE;
    const at::Tensor *table = call.matrix(a[1], c10::kInt), *nodes = call.matrix(a[4], c10::kInt);
    if (!call.ok) Py_RETURN_NONE;
    const int64_t batch = table->size(0);
    const at::Tensor *lens = call.vector(a[2], c10::kInt, batch), *starts = call.vector(a[3], c10::kInt, batch + 1),
                     *kept = call.vector(a[5], c10::kInt, batch);
    const at::Tensor *given = a[6] != Py_None ? call.vector(a[6], c10::kInt, batch) : nullptr;
    if (!call.ok || nodes->size(0) != batch || nodes->size(1) > E2_MAX_DRAFT) Py_RETURN_NONE;
    at::Tensor out;
    try {
        out = given ? *given : call.empty({batch}, c10::kInt);
        e2_keep_args args{};
        args.layers = (int32_t)PyLong_AsLong(PyTuple_GET_ITEM(a[0], 3));
        args.arrays = static_cast<const uint64_t *>(PyLong_AsVoidPtr(PyTuple_GET_ITEM(a[0], 4)));
        args.batch = (int32_t)batch, args.cols = (int32_t)nodes->size(1);
        args.table = data<int32_t>(table), args.table_cols = (int32_t)table->size(1), args.table_stride = Call::stride(*table, table->size(1));
        args.lens = data<int32_t>(lens), args.starts = data<int32_t>(starts), args.kept = data<int32_t>(kept);
        args.nodes = data<int32_t>(nodes), args.nodes_stride = Call::stride(*nodes, nodes->size(1));
        args.lens_out = out.data_ptr<int32_t>();
        if (e2_cache_keep(c, &args, call.stream()) != E2_OK) Py_RETURN_NONE;
    } catch (...) {
        Py_RETURN_NONE;
    }
    return THPVariable_Wrap(std::move(out));
}

PyMethodDef methods[] = {
    {"attend_tree", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(attend_tree)), METH_FASTCALL, nullptr},
    {"verify", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(verify)), METH_FASTCALL, nullptr},
    {"keep", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(keep)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "e2binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_e2binding(void) { return PyModule_Create(&module); }
