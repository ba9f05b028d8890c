// Python entry points of the 4-bit cache and the page bookkeeping (sl.py calls
// them) without ctypes.
//
// The kernels of a small step take 3 to 5 us, so what the host spends per call
// counts: checks of four to nine tensors, the outputs, the descriptor and a ctypes
// call took 4 to 7 us in Python, beside the 3 us of the launch. Here the tensors are
// read directly (append 7.5 us per call -> 3.6, with outputs to make attention 9.9 ->
// 5.3, pages_extend 11.4 -> 5.2).
//
// Every function returns None, with nothing launched, for a call that is not the plain
// case (an argument of another type, shape, layout or device, a device that is not
// the current one, a torch dispatch mode, which is to see the outputs made): sl.py
// then makes the call step by step, which says what is wrong or handles it.
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPGraphsC10Utils.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <ATen/hip/EmptyTensor.h>

#include <numeric>

#include "sl.h"

namespace {

// The library's functions, from the libsl that sl.py loaded.
struct Library {
    decltype(&sl_decode_attn_fp4) attn;
    decltype(&sl_decode_attn_prefix_fp4) attn_prefix;
    decltype(&sl_decode_attn_workspace_size) workspace_size;
    decltype(&sl_decode_attn_prefix_workspace_size) prefix_workspace_size;
    decltype(&sl_kv_append_fp4) append;
    decltype(&sl_kv_write_fp4) write;
    decltype(&sl_kv_read_fp4) read;
    decltype(&sl_pages_extend) extend;
    decltype(&sl_pages_release) release;
} g_lib;

// sl.py's workspaces, {(device, stream, thread): tensor}, its function that makes one, and the one that raises for a status.
PyObject *g_workspaces = nullptr, *g_make_workspace = nullptr, *g_check = nullptr;

constexpr int kPage = 16;
constexpr auto kI32 = at::kInt, kBf16 = at::kBFloat16, kU8 = at::kByte;

// The tensors of one call: all on one device, the current one. `ok` turns false at
// the first that does not fit; its sizes and address are not to be used then.
struct Args {
    bool ok = true;
    int index = -1;   // device

    const at::Tensor *tensor(PyObject *o, at::ScalarType type, int dims)
    {
        if (!ok || !THPVariable_CheckExact(o))
            return fail();
        const at::Tensor &t = THPVariable_Unpack(o);
        if (t.scalar_type() != type || t.dim() != dims || !t.is_cuda() || t.layout() != at::kStrided ||
            !t.is_contiguous())
            return fail();
        const int at = t.get_device();
        if (index < 0 && at == c10::hip::current_device())
            index = at;
        return at == index ? &t : fail();
    }
    // One whose sizes other arguments decide.
    template <class... Sizes>
    void *shaped(PyObject *o, at::ScalarType type, Sizes... sizes)
    {
        const at::Tensor *t = tensor(o, type, (int)sizeof...(sizes));
        if (!t)
            return nullptr;
        int d = 0;
        if (!((t->size(d++) == (int64_t)sizes) && ...)) {
            fail();
            return nullptr;
        }
        return t->data_ptr();
    }
    // The same, or a new one where the caller gave none.
    template <class... Sizes>
    void *output(PyObject *o, at::ScalarType type, at::Tensor &made, Sizes... sizes)
    {
        if (o != Py_None)
            return shaped(o, type, sizes...);
        if (!ok)
            return nullptr;
        made = fresh(type, {(int64_t)sizes...});
        return made.data_ptr();
    }
    at::Tensor fresh(at::ScalarType type, at::IntArrayRef sizes) const
    {
        return at::detail::empty_cuda(sizes, type, at::Device(at::kCUDA, (c10::DeviceIndex)index), std::nullopt);
    }
    // One allocation of int32 for several outputs (some 0.4 us less for each but the first).
    int32_t *parts(std::initializer_list<int64_t> sizes, std::initializer_list<at::Tensor *> made) const
    {
        at::AutoDispatchBelowADInplaceOrView plain;
        const at::Tensor room = fresh(kI32, {std::accumulate(sizes.begin(), sizes.end(), (int64_t)0)});
        int64_t from = 0;
        for (size_t i = 0; i < sizes.size(); from += sizes.begin()[i++])
            *made.begin()[i] = room.as_strided({sizes.begin()[i]}, {1}, from);
        return static_cast<int32_t *>(room.data_ptr());
    }
    hipStream_t stream() const { return c10::hip::getCurrentHIPStream((c10::DeviceIndex)index).stream(); }

private:
    const at::Tensor *fail()
    {
        ok = false;
        return nullptr;
    }
};

// A size that the descriptor's field holds.
bool fits(int64_t n) { return n >= 0 && n <= INT32_MAX; }

bool int_of(PyObject *o, int32_t &x)
{
    if (!PyLong_CheckExact(o))
        return false;
    int overflow = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
    x = (int32_t)v;
    return !overflow && v == x;
}

bool float_of(PyObject *o, float &x)
{
    if (PyFloat_CheckExact(o))
        x = (float)PyFloat_AS_DOUBLE(o);
    return PyFloat_CheckExact(o);
}

PyObject *given(PyObject *o) { return Py_NewRef(o); }
PyObject *result(PyObject *o, const at::Tensor &made) { return o == Py_None ? THPVariable_Wrap(made) : given(o); }

// This thread's workspace on the current stream, at least `bytes`, or one for this call alone if it is being captured
// (both sl.py's to make); undefined, with a Python error, where it could not be made.
at::Tensor workspace(int index, hipStream_t stream, size_t bytes)
{
    const unsigned long long handle = reinterpret_cast<uintptr_t>(stream);
    PyObject *ws = nullptr;
    if (c10::hip::currentStreamCaptureStatusMayInitCtx() == c10::hip::CaptureStatus::None) {
        PyObject *key = Py_BuildValue("(iKk)", index, handle, PyThread_get_thread_ident());
        ws = key ? PyDict_GetItemWithError(g_workspaces, key) : nullptr;
        Py_XDECREF(key);
        if (ws && (size_t)THPVariable_Unpack(ws).numel() >= bytes)
            return THPVariable_Unpack(ws);
    }
    ws = PyErr_Occurred() ? nullptr
                          : PyObject_CallFunction(g_make_workspace, "iKn", index, handle, (Py_ssize_t)bytes);
    if (!ws)
        return {};
    at::Tensor t = THPVariable_Unpack(ws);
    Py_DECREF(ws);
    return t;
}

// A call without the interpreter's lock; false, with a Python error, for a status other than SL_OK.
template <class F>
bool launched(const char *name, F f)
{
    sl_status st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    if (st != SL_OK)
        Py_XDECREF(PyObject_CallFunction(g_check, "is", (int)st, name));
    return st == SL_OK;
}

// None where F says nothing; where it throws too (no memory for an output, a torch error, all
// before a launch): Python makes the call again and meets the same.
template <PyObject *(*F)(PyObject *const *), int ARGS>
PyObject *guarded(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    try {
        PyObject *const r = n == ARGS && !c10::impl::TorchDispatchModeTLS::any_modes_set() ? F(a) : nullptr;
        if (r || PyErr_Occurred())
            return r;
    } catch (...) {
        PyErr_Clear();
    }
    Py_RETURN_NONE;
}

// q, kv_pages, block_table, seq_lens, scale, group_start, shared_pages (None: no prefix sharing), out, num_workers
PyObject *attn(PyObject *const *a)
{
    Args x;
    float scale;
    int32_t workers;
    const at::Tensor *q = x.tensor(a[0], kBf16, 3), *kv = x.tensor(a[1], kU8, 3), *bt = x.tensor(a[2], kI32, 2);
    if (!x.ok || !float_of(a[4], scale) || !int_of(a[8], workers))
        return nullptr;
    const int64_t B = q->size(0), Hq = q->size(1), D = q->size(2), N = kv->size(0), Hkv = kv->size(1),
                  blocks = bt->size(1);
    const int32_t *lens = static_cast<const int32_t *>(x.shaped(a[3], kI32, B));
    const bool prefix = a[6] != Py_None;
    const int32_t *gs = nullptr, *sp = nullptr;
    int64_t ng = 0;
    if (prefix) {
        const at::Tensor *t = x.tensor(a[6], kI32, 1);
        if (!t)
            return nullptr;
        ng = t->size(0);
        sp = static_cast<const int32_t *>(t->data_ptr());
        gs = static_cast<const int32_t *>(x.shaped(a[5], kI32, ng + 1));
    }
    if (!x.ok || kv->size(2) != 17 * D || bt->size(0) != B || B == 0 || !fits(B) || !fits(Hq) || !fits(D) ||
        !fits(N) || !fits(Hkv) || !fits(blocks) || !fits(ng))
        return nullptr;
    at::Tensor made;
    uint16_t *out = static_cast<uint16_t *>(x.output(a[7], kBf16, made, B, Hq, D));
    if (!x.ok)
        return nullptr;
    sl_attn_desc d = {};
    d.batch = (int32_t)B;
    d.num_q_heads = (int32_t)Hq;
    d.num_kv_heads = (int32_t)Hkv;
    d.head_dim = (int32_t)D;
    d.page_size = kPage;
    d.max_blocks_per_seq = (int32_t)blocks;
    d.num_pages = (int32_t)N;
    d.num_workers = workers;
    d.stream = x.stream();
    size_t bytes = 0;
    if ((prefix ? g_lib.prefix_workspace_size(&d, (int32_t)ng, &bytes) : g_lib.workspace_size(&d, &bytes)) != SL_OK)
        return nullptr;
    const at::Tensor ws = workspace(x.index, d.stream, bytes);
    if (!ws.defined())
        return nullptr;
    d.workspace = ws.data_ptr();
    d.workspace_bytes = (size_t)ws.numel();
    const uint16_t *qp = static_cast<const uint16_t *>(q->data_ptr());
    const uint8_t *kp = static_cast<const uint8_t *>(kv->data_ptr());
    const int32_t *tp = static_cast<const int32_t *>(bt->data_ptr());
    const bool done = launched(prefix ? "sl_decode_attn_prefix_fp4" : "sl_decode_attn_fp4", [&] {
        return prefix ? g_lib.attn_prefix(&d, qp, kp, tp, lens, gs, sp, (int32_t)ng, scale, out)
                      : g_lib.attn(&d, qp, kp, tp, lens, scale, out);
    });
    return done ? result(a[7], made) : nullptr;
}

sl_attn_desc pool_desc(const Args &x, int64_t heads, int64_t D, int64_t N)
{
    sl_attn_desc d = {};
    d.num_q_heads = d.num_kv_heads = (int32_t)heads;
    d.head_dim = (int32_t)D;
    d.page_size = kPage;
    d.max_blocks_per_seq = 1;
    d.num_pages = (int32_t)N;
    d.stream = x.stream();
    return d;
}

// k_new, v_new, block_table, seq_lens, kv_pages -> True
PyObject *append(PyObject *const *a)
{
    Args x;
    const at::Tensor *k = x.tensor(a[0], kBf16, 3), *bt = x.tensor(a[2], kI32, 2), *kv = x.tensor(a[4], kU8, 3);
    if (!x.ok)
        return nullptr;
    const int64_t B = k->size(0), H = k->size(1), D = k->size(2), N = kv->size(0), blocks = bt->size(1);
    const uint16_t *v = static_cast<const uint16_t *>(x.shaped(a[1], kBf16, B, H, D));
    const int32_t *lens = static_cast<const int32_t *>(x.shaped(a[3], kI32, B));
    if (!x.ok || kv->size(1) != H || kv->size(2) != 17 * D || bt->size(0) != B || !fits(B) || !fits(H) || !fits(D) ||
        !fits(N) || !fits(blocks))
        return nullptr;
    sl_attn_desc d = pool_desc(x, H, D, N);
    d.batch = (int32_t)B;
    d.max_blocks_per_seq = (int32_t)blocks;
    const bool done = launched("sl_kv_append_fp4", [&] {
        return g_lib.append(&d, static_cast<const uint16_t *>(k->data_ptr()), v,
                            static_cast<const int32_t *>(bt->data_ptr()), lens,
                            static_cast<uint8_t *>(kv->data_ptr()));
    });
    return done ? given(Py_True) : nullptr;
}

// k_new, v_new, slots, kv_pages -> True
PyObject *write(PyObject *const *a)
{
    Args x;
    const at::Tensor *k = x.tensor(a[0], kBf16, 3), *kv = x.tensor(a[3], kU8, 3);
    if (!x.ok)
        return nullptr;
    const int64_t T = k->size(0), H = k->size(1), D = k->size(2), N = kv->size(0);
    const uint16_t *v = static_cast<const uint16_t *>(x.shaped(a[1], kBf16, T, H, D));
    const int32_t *slots = static_cast<const int32_t *>(x.shaped(a[2], kI32, T));
    if (!x.ok || kv->size(1) != H || kv->size(2) != 17 * D || !fits(T) || !fits(H) || !fits(D) || !fits(N))
        return nullptr;
    const sl_attn_desc d = pool_desc(x, H, D, N);
    const bool done = launched("sl_kv_write_fp4", [&] {
        return g_lib.write(&d, static_cast<const uint16_t *>(k->data_ptr()), v, slots, (int32_t)T,
                           static_cast<uint8_t *>(kv->data_ptr()));
    });
    return done ? given(Py_True) : nullptr;
}

// slots, kv_pages, k_out, v_out -> (k, v)
PyObject *read(PyObject *const *a)
{
    Args x;
    const at::Tensor *slots = x.tensor(a[0], kI32, 1), *kv = x.tensor(a[1], kU8, 3);
    if (!x.ok)
        return nullptr;
    const int64_t T = slots->size(0), N = kv->size(0), H = kv->size(1), D = kv->size(2) / 17;
    if (kv->size(2) != 17 * D || !fits(T) || !fits(H) || !fits(D) || !fits(N))
        return nullptr;
    at::Tensor k_made, v_made;
    uint16_t *k = static_cast<uint16_t *>(x.output(a[2], kBf16, k_made, T, H, D));
    uint16_t *v = static_cast<uint16_t *>(x.output(a[3], kBf16, v_made, T, H, D));
    if (!x.ok)
        return nullptr;
    const sl_attn_desc d = pool_desc(x, H, D, N);
    const bool done = launched("sl_kv_read_fp4", [&] {
        return g_lib.read(&d, static_cast<const uint8_t *>(kv->data_ptr()),
                          static_cast<const int32_t *>(slots->data_ptr()), (int32_t)T, k, v);
    });
    return done ? Py_BuildValue("(NN)", result(a[2], k_made), result(a[3], v_made)) : nullptr;
}

sl_attn_desc pages_desc(const Args &x, int64_t B, int64_t blocks, int64_t N)
{
    sl_attn_desc d = pool_desc(x, 1, 64, N);
    d.batch = (int32_t)B;
    d.max_blocks_per_seq = (int32_t)blocks;
    return d;
}

// seq_lens, new_tokens, block_table, free_pages, free_count, max_tokens, seq_lens_out, free_count_out, token_start,
// slots -> (seq_lens_out, token_start, slots, free_count_out)
PyObject *extend(PyObject *const *a)
{
    Args x;
    int32_t most;
    const at::Tensor *lens = x.tensor(a[0], kI32, 1), *bt = x.tensor(a[2], kI32, 2), *free = x.tensor(a[3], kI32, 1);
    if (!x.ok || !int_of(a[5], most) || most < 0)
        return nullptr;
    const int64_t B = lens->size(0), blocks = bt->size(1), N = free->size(0);
    const int32_t *add = static_cast<const int32_t *>(x.shaped(a[1], kI32, B));
    const int32_t *count = static_cast<const int32_t *>(x.shaped(a[4], kI32, 1));
    if (!x.ok || bt->size(0) != B || !fits(B) || !fits(blocks) || !fits(N))
        return nullptr;
    at::Tensor lens_made, count_made, start_made, slots_made;
    int32_t *lens_out, *count_out, *start, *slots;
    if (a[6] == Py_None && a[7] == Py_None && a[8] == Py_None && a[9] == Py_None) {
        int32_t *at = x.parts({B, B + 1, most, 1}, {&lens_made, &start_made, &slots_made, &count_made});
        lens_out = at;
        start = at + B;
        slots = at + 2 * B + 1;
        count_out = slots + most;
    } else {
        lens_out = static_cast<int32_t *>(x.output(a[6], kI32, lens_made, B));
        count_out = static_cast<int32_t *>(x.output(a[7], kI32, count_made, 1));
        start = static_cast<int32_t *>(x.output(a[8], kI32, start_made, B + 1));
        slots = static_cast<int32_t *>(x.output(a[9], kI32, slots_made, most));
    }
    if (!x.ok)
        return nullptr;
    const sl_attn_desc d = pages_desc(x, B, blocks, N);
    const bool done = launched("sl_pages_extend", [&] {
        return g_lib.extend(&d, static_cast<const int32_t *>(lens->data_ptr()), add,
                            static_cast<int32_t *>(bt->data_ptr()), static_cast<const int32_t *>(free->data_ptr()),
                            count, most, lens_out, count_out, start, slots);
    });
    return done ? Py_BuildValue("(NNNN)", result(a[6], lens_made), result(a[8], start_made), result(a[9], slots_made),
                                result(a[7], count_made))
                : nullptr;
}

// finished, seq_lens, block_table, free_pages, free_count, seq_lens_out, free_count_out -> the last two
PyObject *release(PyObject *const *a)
{
    Args x;
    const at::Tensor *lens = x.tensor(a[1], kI32, 1), *bt = x.tensor(a[2], kI32, 2), *free = x.tensor(a[3], kI32, 1);
    if (!x.ok)
        return nullptr;
    const int64_t B = lens->size(0), blocks = bt->size(1), N = free->size(0);
    const int32_t *done_flags = static_cast<const int32_t *>(x.shaped(a[0], kI32, B));
    const int32_t *count = static_cast<const int32_t *>(x.shaped(a[4], kI32, 1));
    if (!x.ok || bt->size(0) != B || !fits(B) || !fits(blocks) || !fits(N))
        return nullptr;
    at::Tensor lens_made, count_made;
    int32_t *lens_out, *count_out;
    if (a[5] == Py_None && a[6] == Py_None) {
        lens_out = x.parts({B, 1}, {&lens_made, &count_made});
        count_out = lens_out + B;
    } else {
        lens_out = static_cast<int32_t *>(x.output(a[5], kI32, lens_made, B));
        count_out = static_cast<int32_t *>(x.output(a[6], kI32, count_made, 1));
    }
    if (!x.ok)
        return nullptr;
    const sl_attn_desc d = pages_desc(x, B, blocks, N);
    const bool done = launched("sl_pages_release", [&] {
        return g_lib.release(&d, done_flags, static_cast<const int32_t *>(lens->data_ptr()),
                             static_cast<const int32_t *>(bt->data_ptr()), static_cast<int32_t *>(free->data_ptr()),
                             count, lens_out, count_out);
    });
    return done ? Py_BuildValue("(NN)", result(a[5], lens_made), result(a[6], count_made)) : nullptr;
}

// bind(addresses of the functions, by name; the workspaces; the function that makes one; the one that raises)
PyObject *bind(PyObject *, PyObject *args)
{
    PyObject *addresses, *workspaces, *make, *check;
    if (!PyArg_ParseTuple(args, "O!O!OO", &PyDict_Type, &addresses, &PyDict_Type, &workspaces, &make, &check))
        return nullptr;
    auto get = [addresses](const char *name, auto &f) {
        PyObject *o = PyDict_GetItemString(addresses, name);
        if (!o) {
            PyErr_Format(PyExc_KeyError, "%s", name);
            return false;
        }
        f = reinterpret_cast<std::decay_t<decltype(f)>>(PyLong_AsVoidPtr(o));
        return !PyErr_Occurred();
    };
    Library lib;
    if (!get("sl_decode_attn_fp4", lib.attn) || !get("sl_decode_attn_prefix_fp4", lib.attn_prefix) ||
        !get("sl_decode_attn_workspace_size", lib.workspace_size) ||
        !get("sl_decode_attn_prefix_workspace_size", lib.prefix_workspace_size) ||
        !get("sl_kv_append_fp4", lib.append) || !get("sl_kv_write_fp4", lib.write) ||
        !get("sl_kv_read_fp4", lib.read) || !get("sl_pages_extend", lib.extend) ||
        !get("sl_pages_release", lib.release))
        return nullptr;
    g_lib = lib;
    g_workspaces = given(workspaces);
    g_make_workspace = given(make);
    g_check = given(check);
    Py_RETURN_NONE;
}

template <PyObject *(*F)(PyObject *const *), int ARGS>
PyMethodDef entry(const char *name)
{
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(guarded<F, ARGS>)), METH_FASTCALL, nullptr};
}
PyMethodDef g_methods[] = {entry<attn, 9>("attn"),      entry<append, 5>("append"),   entry<write, 4>("write"),
                           entry<read, 4>("read"),      entry<extend, 10>("extend"),  entry<release, 7>("release"),
                           {"bind", bind, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};

PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&g_module); }
