// The tensor entry points of the Python package (sdpa, sdpa_kv, sdpa_paged, sdpa_backward, sdpa_tree, sdpa_tree_paged, and those
// around attention: tree_mask, cache_step, qk_norm_rope, qk_norm_rope_cache, qk_norm_rope_backward) in native code: argument
// checks, output and workspace tensors from torch's allocator, the current stream, and one call into the C-ABI of include/tiled_sdpa.h.
//
// Why native: a short call is bound by the host.  One forward call of a small problem (B=1 H=2 S=128 D=64, a kernel of
// 4.4 us) took 8.7 us of host time through Python attribute reads, data_ptr() calls and ctypes argument conversion, a
// decoding step with splits (two kernels, a workspace query, two allocations) 17.5 us, a backward call 22-28 us.  The
// same calls take 5.1, 8.6 and 12-17 us here; most of what is left is the launches.
//
// Each function takes every argument of its Python wrapper by position and returns the result object, or the status
// code (a Python int) of a call that the library refused; the wrapper turns that into TiledSdpaError.
#include <Python.h>

#include <cmath>
#include <limits>

#include <ATen/core/Tensor.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "rows_overlap.h"
#include "tiled_sdpa.h"

namespace {

// thrown with a Python error set
struct PyFail {};

[[noreturn]] void fail(const char *text)
{
    PyErr_SetString(PyExc_ValueError, text);
    throw PyFail{};
}

[[noreturn]] void fail_named(const char *name, const char *text)
{
    PyErr_Format(PyExc_ValueError, "%s %s", name, text);
    throw PyFail{};
}

// Tensor arguments are borrowed from the caller's references; THPVariable_Unpack only looks inside.
const at::Tensor &device_tensor(PyObject *obj, const char *name)
{
    if (!THPVariable_Check(obj)) fail_named(name, "must be a device tensor");
    const at::Tensor &t = THPVariable_Unpack(obj);
    if (!t.is_cuda()) fail_named(name, "must be a device tensor");
    return t;
}

const at::Tensor &heads_tensor(PyObject *obj, const char *name)
{
    const at::Tensor &t = device_tensor(obj, name);
    if (t.dim() != 4 || !t.is_contiguous()) fail_named(name, "must be contiguous [B, H, S, D]");
    return t;
}

int element_type(const at::Tensor &t)
{
    if (t.scalar_type() == at::kHalf) return TSDPA_F16;
    if (t.scalar_type() == at::kBFloat16) return TSDPA_BF16;
    fail("dtype must be float16 or bfloat16");
}

void same_type(const at::Tensor &q, const at::Tensor &k, const at::Tensor &v)
{
    if ((q.scalar_type() != at::kHalf && q.scalar_type() != at::kBFloat16) || k.scalar_type() != q.scalar_type() ||
        v.scalar_type() != q.scalar_type())
        fail("q, k, v must share dtype float16 or bfloat16");
}

int as_int(PyObject *obj)
{
    const long x = PyLong_AsLong(obj);
    if (x == -1 && PyErr_Occurred()) throw PyFail{};
    if (x < std::numeric_limits<int>::min() || x > std::numeric_limits<int>::max()) {
        PyErr_SetString(PyExc_OverflowError, "argument does not fit a 32-bit integer");
        throw PyFail{};
    }
    return (int)x;
}

bool as_bool(PyObject *obj)
{
    const int x = PyObject_IsTrue(obj);
    if (x < 0) throw PyFail{};
    return x != 0;
}

unsigned as_flags(PyObject *flags, PyObject *causal)
{
    const unsigned long x = PyLong_AsUnsignedLongMask(flags);
    if (x == (unsigned long)-1 && PyErr_Occurred()) throw PyFail{};
    return (unsigned)x | (as_bool(causal) ? (unsigned)TSDPA_FLAG_CAUSAL : 0u);
}

float as_scale(PyObject *obj)
{
    if (obj == Py_None) return std::numeric_limits<float>::quiet_NaN();
    const double x = PyFloat_AsDouble(obj);
    if (x == -1.0 && PyErr_Occurred()) throw PyFail{};
    return (float)x;
}

struct Tile { int m = 0, n = 0; };

Tile as_tile(PyObject *obj)
{
    Tile t;
    if (obj == Py_None) return t;
    PyObject *seq = PySequence_Fast(obj, "tile must be (tile_m, tile_n)");
    if (!seq) throw PyFail{};
    if (PySequence_Fast_GET_SIZE(seq) != 2) {
        Py_DECREF(seq);
        fail("tile must be (tile_m, tile_n)");
    }
    PyObject *const *items = PySequence_Fast_ITEMS(seq);
    try {
        t.m = as_int(items[0]);
        t.n = as_int(items[1]);
    } catch (...) {
        Py_DECREF(seq);
        throw;
    }
    Py_DECREF(seq);
    return t;
}

// Lets other Python threads run while the allocator or the launch may block (a full queue, say, that waits for a host function
// of another thread).
struct NoGil {
    PyThreadState *state = PyEval_SaveThread();
    ~NoGil() { PyEval_RestoreThread(state); }
};

at::Tensor empty(at::IntArrayRef size, at::ScalarType type, const at::Tensor &like)
{
    const NoGil without;
    return at::Tensor(at::detail::empty_cuda(size, type, like.device(), std::nullopt));
}

// Makes the tensors' device current for the call if it is not, and names the stream that is current on it.
struct Launch {
    c10::OptionalDeviceGuard guard;
    void *stream;
    explicit Launch(const at::Tensor &q)
    {
        const c10::DeviceIndex index = q.device().index();
        if (c10::hip::current_device() != index) guard.reset_device(q.device());
        stream = (void *)c10::hip::getCurrentHIPStream(index).stream();
    }
};

// (the arguments are evaluated before the lock is let go)
template <typename... P, typename... A> int without_gil(int (*call)(P...), A... args)
{
    const NoGil without;
    return call(args...);
}

void *data(const at::Tensor &t) { return t.data_ptr(); }

bool same_sizes(const at::Tensor &a, const at::Tensor &b) { return a.sizes() == b.sizes(); }

// `out` of the caller, checked against `like`, or a new tensor of that shape
at::Tensor output(PyObject *obj, const at::Tensor &like, const char *complaint)
{
    if (obj == Py_None) return empty(like.sizes(), like.scalar_type(), like);
    if (!THPVariable_Check(obj)) fail(complaint);
    const at::Tensor &t = THPVariable_Unpack(obj);
    if (!same_sizes(t, like) || t.scalar_type() != like.scalar_type() || !t.is_contiguous() || t.device() != like.device())
        fail(complaint);
    return t;
}

// The object to hand back for a tensor: the caller's own if they passed one.
PyObject *give(PyObject *passed, const at::Tensor &t)
{
    if (passed != Py_None) {
        Py_INCREF(passed);
        return passed;
    }
    return THPVariable_Wrap(t);
}

PyObject *result(int status, PyObject *out_obj, const at::Tensor &out, bool with_lse, PyObject *lse_obj, const at::Tensor &lse)
{
    if (status != TSDPA_OK) return PyLong_FromLong(status);
    PyObject *o = give(out_obj, out);
    if (!o || !with_lse) return o;
    PyObject *l = give(lse_obj, lse);
    if (!l) {
        Py_DECREF(o);
        return nullptr;
    }
    PyObject *pair = PyTuple_New(2);
    if (!pair) {
        Py_DECREF(o);
        Py_DECREF(l);
        return nullptr;
    }
    PyTuple_SET_ITEM(pair, 0, o);
    PyTuple_SET_ITEM(pair, 1, l);
    return pair;
}

struct Workspace {
    at::Tensor held;
    void *ptr = nullptr;
    unsigned long long bytes = 0;
    Workspace() = default;
    // the caller's buffer, or `need` bytes of torch's.  The kernels write to it as to one range of bytes: it has to be that,
    // and on the device of the call (of a call that needs none it is not looked at)
    Workspace(PyObject *obj, unsigned long long need, const at::Tensor &like)
    {
        if (obj != Py_None) {
            if (!THPVariable_Check(obj)) fail("workspace must be a device tensor");
            held = THPVariable_Unpack(obj);
            if (need > 0 && (held.device() != like.device() || !held.is_non_overlapping_and_dense()))
                fail("workspace must be a dense tensor on the device of q");
        } else if (need > 0) {
            held = empty({(int64_t)need}, at::kByte, like);
        } else {
            return;
        }
        ptr = data(held);
        bytes = (unsigned long long)held.numel() * held.element_size();
    }
};

void need_args(Py_ssize_t got, Py_ssize_t want)
{
    if (got == want) return;
    PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", want, got);
    throw PyFail{};
}

// Runs a function body; C++ exceptions (torch's allocator out of memory among them) become Python's.
template <typename F> PyObject *guarded(F &&body)
{
    try {
        return body();
    } catch (const PyFail &) {
        return nullptr;
    } catch (...) {
        return torch::translate_exception_to_python(std::current_exception()), nullptr;
    }
}

// sdpa(q, k, v, causal, scale, return_lse, out, lse_out, tile, flags)
PyObject *call_sdpa(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        need_args(n, 10);
        const at::Tensor &q = heads_tensor(args[0], "q"), &k = heads_tensor(args[1], "k"), &v = heads_tensor(args[2], "v");
        const unsigned flags = as_flags(args[9], args[3]);
        const float scale = as_scale(args[4]);
        const bool with_lse = as_bool(args[5]);
        const Tile tile = as_tile(args[8]);
        same_type(q, k, v);
        if (!same_sizes(q, k) || !same_sizes(q, v) || k.device() != q.device() || v.device() != q.device())
            fail("q, k, v must have identical shape and device");
        const at::IntArrayRef s = q.sizes();
        at::Tensor out = output(args[6], q, "out must match q in shape, dtype, device and be contiguous");
        at::Tensor lse;
        if (with_lse) {
            if (args[7] != Py_None) {
                static const char text[] = "lse_out must be contiguous float32 [B, H, S] on the device of q";
                if (!THPVariable_Check(args[7])) fail(text);
                lse = THPVariable_Unpack(args[7]);
                if (lse.sizes() != s.slice(0, 3) || lse.scalar_type() != at::kFloat || !lse.is_contiguous() || lse.device() != q.device())
                    fail(text);
            } else {
                lse = empty(s.slice(0, 3), at::kFloat, q);
            }
        }
        const Launch on(q);
        const int st = without_gil(tiled_sdpa_fwd_ex, data(q), data(k), data(v), data(out), with_lse ? (float *)data(lse) : nullptr,
                                         (int)s[0], (int)s[1], (int)s[2], (int)s[3], scale, element_type(q), on.stream,
                                         tile.m, tile.n, flags);
        return result(st, args[6], out, with_lse, args[7], lse);
    });
}

// The split count of a call that leaves it to the library (which sees B * Hkv heads of G * Sq rows each).  A tile that the library
// does not offer is for the call itself to refuse, after the checks that come before that one.
int heuristic_splits(int B, int H, int Hkv, int Sq, int Skv, int D, int dtype, unsigned flags, bool drop_causal, Tile tile, int *splits)
{
    const int st = tiled_sdpa_kv_tile_splits(B, Hkv, (int)((int64_t)(H / Hkv) * Sq), Skv, D, dtype,
                                             drop_causal ? flags & ~(unsigned)TSDPA_FLAG_CAUSAL : flags, tile.m, tile.n, splits);
    return st == TSDPA_ERR_BAD_TILE ? TSDPA_OK : st;
}

// sdpa_kv(q, k, v, causal, scale, splits, return_lse, out, workspace, tile, flags, kv_lens)
PyObject *call_sdpa_kv(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        need_args(n, 12);
        const at::Tensor &q = heads_tensor(args[0], "q"), &k = heads_tensor(args[1], "k"), &v = heads_tensor(args[2], "v");
        const unsigned flags = as_flags(args[10], args[3]);
        const float scale = as_scale(args[4]);
        int splits = args[5] == Py_None ? 0 : as_int(args[5]);
        const bool with_lse = as_bool(args[6]);
        const Tile tile = as_tile(args[9]);
        same_type(q, k, v);
        const at::IntArrayRef s = q.sizes(), t = k.sizes();
        if (!same_sizes(k, v) || s[0] != t[0] || s[3] != t[3]) fail("q must be [B, H, Sq, D] and k, v [B, Hkv, Skv, D]");
        if (t[1] == 0 || s[1] % t[1] != 0) fail("the number of query heads must be a multiple of the number of key/value heads");
        if (k.device() != q.device() || v.device() != q.device()) fail("q, k, v must be on one device");
        const int *lens = nullptr;
        if (args[11] != Py_None) {
            static const char text[] = "kv_lens must be a contiguous int32 tensor [B] on the device of q";
            if (!THPVariable_Check(args[11])) fail(text);
            const at::Tensor &l = THPVariable_Unpack(args[11]);
            if (l.scalar_type() != at::kInt || l.device() != q.device() || l.dim() != 1 || l.size(0) != s[0] || !l.is_contiguous())
                fail(text);
            lens = (const int *)data(l);
        }
        const int B = (int)s[0], H = (int)s[1], Sq = (int)s[2], D = (int)s[3], Hkv = (int)t[1], Skv = (int)t[2];
        const int dtype = element_type(q);
        at::Tensor out = output(args[7], q, "out must match q in shape, dtype, device and be contiguous"), lse;
        if (with_lse) lse = empty(s.slice(0, 3), at::kFloat, q);
        const bool heuristic = splits == 0;
        if (heuristic) {
            const int st = heuristic_splits(B, H, Hkv, Sq, Skv, D, dtype, flags, H != Hkv, tile, &splits);
            if (st != TSDPA_OK) return PyLong_FromLong(st);
        }
        const Workspace ws(args[8], tiled_sdpa_kv_workspace_bytes(B, H, Sq, D, splits), q);
        if (heuristic && args[8] != Py_None) splits = 0;      // (what fits the caller's buffer: the library decides)
        const Launch on(q);
        const int st = without_gil(tiled_sdpa_fwd_kvcache, data(q), data(k), data(v), data(out), with_lse ? (float *)data(lse) : nullptr, lens,
                                              B, H, Hkv, Sq, Skv, D, scale, dtype, on.stream, tile.m, tile.n, flags, splits,
                                              ws.ptr, ws.bytes);
        return result(st, args[7], out, with_lse, Py_None, lse);
    });
}

// sdpa_paged(q, k_pages, v_pages, kv_lens, block_table, causal, scale, splits, return_lse, out, workspace, tile, flags)
PyObject *call_sdpa_paged(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        need_args(n, 13);
        const at::Tensor *tensors[3];
        static const char *names[3] = {"q", "k_pages", "v_pages"};
        for (int i = 0; i < 3; ++i) {
            if (!THPVariable_Check(args[i])) fail_named(names[i], "must be a contiguous 4-d device tensor");
            tensors[i] = &THPVariable_Unpack(args[i]);
            if (!tensors[i]->is_cuda() || tensors[i]->dim() != 4 || !tensors[i]->is_contiguous())
                fail_named(names[i], "must be a contiguous 4-d device tensor");
        }
        const at::Tensor &q = *tensors[0], &k = *tensors[1], &v = *tensors[2];
        const unsigned flags = as_flags(args[12], args[5]);
        const float scale = as_scale(args[6]);
        int splits = args[7] == Py_None ? 0 : as_int(args[7]);
        const bool with_lse = as_bool(args[8]);
        const Tile tile = as_tile(args[11]);
        if ((q.scalar_type() != at::kHalf && q.scalar_type() != at::kBFloat16) || k.scalar_type() != q.scalar_type() ||
            v.scalar_type() != q.scalar_type())
            fail("q, k_pages, v_pages must share dtype float16 or bfloat16");
        const at::IntArrayRef s = q.sizes(), t = k.sizes();
        if (!same_sizes(k, v) || t[3] != s[3] || k.device() != q.device() || v.device() != q.device())
            fail("k_pages, v_pages must be [P, Hkv, block_rows, D] on the device of q");
        if (t[1] == 0 || s[1] % t[1] != 0) fail("the number of query heads must be a multiple of the number of key/value heads");
        if (!THPVariable_Check(args[3])) fail("kv_lens must be a contiguous int32 device tensor");
        if (!THPVariable_Check(args[4])) fail("block_table must be a contiguous int32 device tensor");
        const at::Tensor &lens = THPVariable_Unpack(args[3]), &table = THPVariable_Unpack(args[4]);
        if (lens.scalar_type() != at::kInt || lens.device() != q.device() || !lens.is_contiguous() || lens.dim() != 1 || lens.size(0) != s[0])
            fail("kv_lens must be a contiguous int32 device tensor");
        if (table.scalar_type() != at::kInt || table.device() != q.device() || !table.is_contiguous())
            fail("block_table must be a contiguous int32 device tensor");
        if (table.dim() != 2 || table.size(0) != s[0]) fail("block_table must be [B, max_blocks]");
        const int B = (int)s[0], H = (int)s[1], Sq = (int)s[2], D = (int)s[3], Hkv = (int)t[1], block_rows = (int)t[2];
        const int max_blocks = (int)table.size(1), dtype = element_type(q);
        at::Tensor out = output(args[9], q, "out must match q in shape, dtype, device and be contiguous"), lse;
        if (with_lse) lse = empty(s.slice(0, 3), at::kFloat, q);
        const bool heuristic = splits == 0;
        if (heuristic) {
            const int64_t rows = (int64_t)max_blocks * block_rows;
            if (rows > std::numeric_limits<int>::max()) return PyLong_FromLong(TSDPA_ERR_BAD_SHAPE);
            const int st = heuristic_splits(B, H, Hkv, Sq, rows > 1 ? (int)rows : 1, D, dtype, flags, true, tile, &splits);
            if (st != TSDPA_OK) return PyLong_FromLong(st);
        }
        const Workspace ws(args[10], tiled_sdpa_kv_workspace_bytes(B, H, Sq, D, splits), q);
        if (heuristic && args[10] != Py_None) splits = 0;
        const Launch on(q);
        const int st = without_gil(tiled_sdpa_fwd_paged, data(q), data(k), data(v), data(out), with_lse ? (float *)data(lse) : nullptr,
                                            (const int *)data(lens), (const int *)data(table), B, H, Hkv, Sq, max_blocks,
                                            block_rows, D, scale, dtype, on.stream, tile.m, tile.n, flags, splits, ws.ptr, ws.bytes);
        return result(st, args[9], out, with_lse, Py_None, lse);
    });
}

// sdpa_backward(q, k, v, o, dout, lse, causal, scale, workspace, grads)
PyObject *call_sdpa_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        need_args(n, 10);
        const at::Tensor &q = heads_tensor(args[0], "q"), &k = heads_tensor(args[1], "k"), &v = heads_tensor(args[2], "v");
        const at::Tensor &o = heads_tensor(args[3], "o"), &dout = heads_tensor(args[4], "dout");
        auto agree = [&](const at::Tensor &t, const at::Tensor &like) {
            if (!same_sizes(t, like) || t.scalar_type() != q.scalar_type() || t.device() != q.device())
                fail("q, o, dout and k, v must agree in shape, dtype and device");
        };
        agree(k, k);
        agree(v, k);
        agree(o, q);
        agree(dout, q);
        const int dtype = element_type(q);
        const at::IntArrayRef s = q.sizes(), t = k.sizes();
        if (t[0] != s[0] || t[2] != s[2] || t[3] != s[3] || t[1] == 0 || s[1] % t[1] != 0)
            fail("k, v must be [B, Hkv, S, D] with H a multiple of Hkv");
        if (!THPVariable_Check(args[5])) fail("lse must be contiguous float32 [B, H, S] on the same device");
        const at::Tensor &lse = THPVariable_Unpack(args[5]);
        if (lse.sizes() != s.slice(0, 3) || lse.scalar_type() != at::kFloat || !lse.is_contiguous() || lse.device() != q.device())
            fail("lse must be contiguous float32 [B, H, S] on the same device");
        const unsigned flags = as_bool(args[6]) ? (unsigned)TSDPA_FLAG_CAUSAL : 0u;
        const float scale = as_scale(args[7]);
        at::Tensor grad[3];
        if (args[9] == Py_None) {
            grad[0] = empty(s, q.scalar_type(), q);
            grad[1] = empty(t, q.scalar_type(), q);
            grad[2] = empty(t, q.scalar_type(), q);
        } else {
            static const char *complaints[3] = {"dq must match q in shape, dtype, device and be contiguous",
                                                "dk must match k in shape, dtype, device and be contiguous",
                                                "dv must match k in shape, dtype, device and be contiguous"};
            PyObject *seq = PySequence_Fast(args[9], "grads must be (dq, dk, dv)");
            if (!seq) throw PyFail{};
            if (PySequence_Fast_GET_SIZE(seq) < 3) {
                Py_DECREF(seq);
                fail("grads must be (dq, dk, dv)");
            }
            try {
                for (int i = 0; i < 3; ++i) {
                    PyObject *item = PySequence_Fast_GET_ITEM(seq, i);
                    if (item == Py_None) fail(complaints[i]);
                    grad[i] = output(item, i == 0 ? q : k, complaints[i]);
                }
            } catch (...) {
                Py_DECREF(seq);
                throw;
            }
            Py_DECREF(seq);
        }
        const int B = (int)s[0], H = (int)s[1], S = (int)s[2], D = (int)s[3];
        const unsigned long long least = tiled_sdpa_bwd_workspace_bytes(B, H, S);
        Workspace ws;
        if (args[8] == Py_None) {
            // Without memory for the sums of dQ the call takes the passes that need none, as it did before there were such sums.  (Whatever the
            // allocator's error: without its cache it reports HIP's own.  One that is not about the size comes again.)
            const unsigned long long full = tiled_sdpa_bwd_full_workspace_bytes(B, H, (int)t[1], S, D, flags);
            try {
                ws = Workspace(args[8], full, q);
            } catch (const c10::Error &) {
                if (full == least) throw;
            }
        }
        if (!ws.ptr) ws = Workspace(args[8], least, q);
        const Launch on(q);
        const int st = without_gil(tiled_sdpa_bwd_gqa, data(q), data(k), data(v), data(o), data(dout), (const float *)data(lse), data(grad[0]),
                                          data(grad[1]), data(grad[2]), B, H, (int)t[1], S, D, scale, dtype, flags, ws.ptr,
                                          ws.bytes, on.stream);
        if (st != TSDPA_OK) return PyLong_FromLong(st);
        if (args[9] != Py_None) {
            Py_INCREF(args[9]);
            return args[9];
        }
        PyObject *all = PyTuple_New(3);
        if (!all) return nullptr;
        for (int i = 0; i < 3; ++i) {
            PyObject *g = THPVariable_Wrap(grad[i]);
            if (!g) {
                Py_DECREF(all);
                return nullptr;
            }
            PyTuple_SET_ITEM(all, i, g);
        }
        return all;
    });
}

// An int32 tensor on the device of `like`, contiguous, of the given shape.
const int *int_data(PyObject *obj, at::IntArrayRef shape, const at::Device &device, const char *complaint)
{
    if (!THPVariable_Check(obj)) fail(complaint);
    const at::Tensor &t = THPVariable_Unpack(obj);
    if (t.scalar_type() != at::kInt || t.device() != device || t.sizes() != shape || !t.is_contiguous()) fail(complaint);
    return (const int *)data(t);
}

// The mask of a tree: int64 [T, W] for all entries, or [B, T, W].
struct TreeMask { const long long *data; long long batch; };
TreeMask tree_mask_of(PyObject *obj, int64_t B, int64_t T, const at::Tensor &q)
{
    static const char text[] = "mask must be a contiguous int64 tensor [T, ceil(T / 64)] or [B, T, ceil(T / 64)] on the device of q";
    if (!THPVariable_Check(obj)) fail(text);
    const at::Tensor &m = THPVariable_Unpack(obj);
    const int64_t W = (T + 63) / 64;
    if (m.scalar_type() != at::kLong || m.device() != q.device() || !m.is_contiguous() || (m.dim() != 2 && m.dim() != 3)) fail(text);
    const at::IntArrayRef s = m.sizes();
    if (s[s.size() - 2] != T || s[s.size() - 1] != W || (m.dim() == 3 && s[0] != B)) fail(text);
    return TreeMask{(const long long *)data(m), m.dim() == 3 ? (long long)(T * W) : 0};
}

// sdpa_tree(q, k, v, kv_lens, block_table, mask, scale, splits, return_lse, out, workspace): dense (block_table None, kv_lens may be) or paged
PyObject *call_sdpa_tree(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        need_args(n, 11);
        const at::Tensor &q = heads_tensor(args[0], "q"), &k = heads_tensor(args[1], "k"), &v = heads_tensor(args[2], "v");
        const bool paged = args[4] != Py_None;
        const float scale = as_scale(args[6]);
        int splits = args[7] == Py_None ? 0 : as_int(args[7]);
        const bool with_lse = as_bool(args[8]);
        same_type(q, k, v);
        const at::IntArrayRef s = q.sizes(), t = k.sizes();
        if (!same_sizes(k, v) || s[3] != t[3] || (!paged && s[0] != t[0]))
            fail(paged ? "k_pages, v_pages must be [P, Hkv, block_rows, D]" : "q must be [B, H, T, D] and k, v [B, Hkv, Skv, D]");
        if (t[1] == 0 || s[1] % t[1] != 0) fail("the number of query heads must be a multiple of the number of key/value heads");
        if (k.device() != q.device() || v.device() != q.device()) fail("q, k, v must be on one device");
        const int *lens = nullptr, *table = nullptr;
        if (paged || args[3] != Py_None) lens = int_data(args[3], s.slice(0, 1), q.device(), "kv_lens must be a contiguous int32 tensor [B] on the device of q");
        const int B = (int)s[0], H = (int)s[1], T = (int)s[2], D = (int)s[3], Hkv = (int)t[1], dtype = element_type(q);
        int max_blocks = 0;
        int64_t cap = t[2];
        if (paged) {
            static const char text[] = "block_table must be a contiguous int32 tensor [B, max_blocks] on the device of q";
            if (!THPVariable_Check(args[4])) fail(text);
            const at::Tensor &x = THPVariable_Unpack(args[4]);
            if (x.dim() != 2) fail(text);
            table = int_data(args[4], {s[0], x.size(1)}, q.device(), text);
            if (x.size(1) > std::numeric_limits<int>::max()) return PyLong_FromLong(TSDPA_ERR_BAD_SHAPE);
            max_blocks = (int)x.size(1);
            cap = (int64_t)max_blocks * t[2];
        }
        if (cap > std::numeric_limits<int>::max()) return PyLong_FromLong(TSDPA_ERR_BAD_SHAPE);
        const TreeMask mask = tree_mask_of(args[5], s[0], s[2], q);
        at::Tensor out = output(args[9], q, "out must match q in shape, dtype, device and be contiguous"), lse;
        if (with_lse) lse = empty(s.slice(0, 3), at::kFloat, q);
        const bool heuristic = splits == 0;
        if (heuristic) {
            const int st = tiled_sdpa_tree_default_splits(B, H, Hkv, T, (int)cap, D, dtype, &splits);
            if (st != TSDPA_OK) return PyLong_FromLong(st);
        }
        const Workspace ws(args[10], tiled_sdpa_kv_workspace_bytes(B, H, T, D, splits), q);
        if (heuristic && args[10] != Py_None) splits = 0;
        const Launch on(q);
        float *const lse_data = with_lse ? (float *)data(lse) : nullptr;
        const int st = paged ? without_gil(tiled_sdpa_fwd_tree_paged, data(q), data(k), data(v), data(out), lse_data, lens, table, mask.data, mask.batch,
                                           B, H, Hkv, T, max_blocks, (int)t[2], D, scale, dtype, on.stream, splits, ws.ptr, ws.bytes)
                             : without_gil(tiled_sdpa_fwd_tree, data(q), data(k), data(v), data(out), lse_data, lens, mask.data, mask.batch,
                                           B, H, Hkv, T, (int)cap, D, scale, dtype, on.stream, splits, ws.ptr, ws.bytes);
        return result(st, args[9], out, with_lse, Py_None, lse);
    });
}

// A tuple of the tensors given, or the status code.
PyObject *tuple_of(int status, std::initializer_list<const at::Tensor *> tensors)
{
    if (status != TSDPA_OK) return PyLong_FromLong(status);
    PyObject *all = PyTuple_New((Py_ssize_t)tensors.size());
    if (!all) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor *t : tensors) {
        PyObject *obj;
        if (t->defined()) {
            obj = THPVariable_Wrap(*t);
        } else {
            Py_INCREF(Py_None);
            obj = Py_None;
        }
        if (!obj) {
            Py_DECREF(all);
            return nullptr;
        }
        PyTuple_SET_ITEM(all, i++, obj);
    }
    return all;
}

// The objects of a caller's tuple of `count`, given to `take` one after another (which keeps what it needs of them: a sequence made for
// the call ends here).
template <typename F> void each_of(PyObject *obj, Py_ssize_t count, const char *complaint, F &&take)
{
    PyObject *seq = PySequence_Fast(obj, complaint);
    if (!seq) throw PyFail{};
    try {
        if (PySequence_Fast_GET_SIZE(seq) != count) fail(complaint);
        for (Py_ssize_t i = 0; i < count; ++i) take(i, PySequence_Fast_GET_ITEM(seq, i));
    } catch (...) {
        Py_DECREF(seq);
        throw;
    }
    Py_DECREF(seq);
}

// The tensors of a caller's tuple, or undefined ones.
template <int N> struct Given {
    at::Tensor t[N];
    Given(PyObject *obj, const char *complaint)
    {
        if (obj == Py_None) return;
        each_of(obj, N, complaint, [&](Py_ssize_t i, PyObject *x) {
            if (!THPVariable_Check(x)) fail(complaint);
            t[i] = THPVariable_Unpack(x);
        });
    }
};

// New tensors that share one allocation, each at a multiple of 64 bytes of it (four allocations of a few bytes take 2.5 us, more than the
// kernel that fills them).
class Carver {
    c10::Storage storage;
    int64_t at = 0;

public:
    static int64_t room(int64_t count, int64_t size) { return (count * size + 63) / 64 * 64; }
    Carver(int64_t bytes, const at::Tensor &like) : storage(empty({bytes}, at::kByte, like).storage()) {}
    at::Tensor next(at::IntArrayRef shape, at::ScalarType type)
    {
        at::Tensor t = at::detail::make_tensor<at::TensorImpl>(c10::Storage(storage), c10::DispatchKeySet(c10::DispatchKey::CUDA), c10::scalarTypeToTypeMeta(type));
        const int64_t size = c10::elementSize(type);
        t.unsafeGetTensorImpl()->set_storage_offset(at / size);
        t.unsafeGetTensorImpl()->set_sizes_contiguous(shape);
        at += room(t.numel(), size);
        return t;
    }
};

// An output of the caller's, or a new tensor.
at::Tensor made(const at::Tensor &t, at::IntArrayRef shape, at::ScalarType type, const at::Tensor &like, const char *complaint)
{
    if (!t.defined()) return empty(shape, type, like);
    if (t.sizes() != shape || t.scalar_type() != type || !t.is_contiguous() || t.device() != like.device()) fail(complaint);
    return t;
}

// Memory of a tensor: contiguous, or rows of a strided one ([B, S, heads, D]).  Outputs that overlap what a kernel's other workgroups
// still read are refused; most calls' tensors are told apart by where they begin and end.
struct Extent {
    int64_t at = 0, end = 0;
    const at::Tensor *rows = nullptr;              // strided
    Extent() = default;
    explicit Extent(const at::Tensor &t) : at((int64_t)(uintptr_t)data(t)), end(at + (int64_t)t.nbytes())
    {
        if (t.dim() != 4 || end == at || t.is_contiguous()) return;
        rows = &t;
        end = at + (int64_t)t.element_size() * (t.stride(0) * (t.size(0) - 1) + t.stride(1) * (t.size(1) - 1) + t.stride(2) * (t.size(2) - 1) + t.size(3));
    }
    Extent(const void *p, int64_t bytes) : at((int64_t)(uintptr_t)p), end(p ? at + bytes : at) {}
    Extent(const int *p, int64_t count) : Extent((const void *)p, count * (int64_t)sizeof(int)) {}
    tsdpa::RowSet set() const
    {
        if (!rows) return tsdpa::RowSet{at, end - at};
        const int64_t size = (int64_t)rows->element_size();
        tsdpa::RowSet r{at, rows->size(3) * size, 3};
        for (int i = 0; i < 3; ++i) r.dim[i] = {rows->stride(i) * size, rows->size(i)};
        return r;
    }
    bool meets(const Extent &o) const
    {
        if (at >= o.end || o.at >= end || at == end || o.at == o.end) return false;
        return (!rows && !o.rows) || tsdpa::RowsOverlap()(set(), o.set());
    }
};
void distinct(std::initializer_list<Extent> outputs, std::initializer_list<Extent> inputs, const char *complaint)
{
    for (const Extent *o = outputs.begin(); o != outputs.end(); ++o) {
        for (const Extent &i : inputs)
            if (o->meets(i)) fail(complaint);
        for (const Extent *other = outputs.begin(); other != o; ++other)
            if (o->meets(*other)) fail(complaint);
    }
}

// tree_mask(parents, out)
PyObject *call_tree_mask(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        need_args(n, 2);
        const at::Tensor &parents = device_tensor(args[0], "parents");
        if (parents.scalar_type() != at::kInt || !parents.is_contiguous() || (parents.dim() != 1 && parents.dim() != 2))
            fail("parents must be contiguous int32 [T] or [B, T]");
        const at::IntArrayRef s = parents.sizes();
        const int64_t T = s[s.size() - 1], B = s.size() == 2 ? s[0] : 1;
        if (T > 1024 || B > std::numeric_limits<int>::max()) return PyLong_FromLong(TSDPA_ERR_BAD_SHAPE);
        const int64_t words[3] = {B, T, (T + 63) / 64};
        const at::IntArrayRef shape(s.size() == 2 ? words : words + 1, s.size() + 1);
        static const char text[] = "out must be (mask, depths): contiguous int64 [..., T, ceil(T / 64)] and int32 [..., T] on the device of parents";
        at::Tensor mask, depths;
        if (args[1] == Py_None) {
            Carver carve(Carver::room(B * T * words[2], 8) + Carver::room(B * T, 4), parents);
            mask = carve.next(shape, at::kLong);
            depths = carve.next(s, at::kInt);
        } else {
            const Given<2> given(args[1], text);
            mask = made(given.t[0], shape, at::kLong, parents, text);
            depths = made(given.t[1], s, at::kInt, parents, text);
            distinct({Extent(mask), Extent(depths)}, {Extent(parents)}, "mask, depths and parents must not overlap");
        }
        const Launch on(parents);
        const int st = without_gil(tiled_sdpa_tree_mask, (const int *)data(parents), (long long *)data(mask), (int *)data(depths), (int)B, (int)T, on.stream);
        return tuple_of(st, {&mask, &depths});
    });
}

// cache_step(kv_lens, counts, S, block_rows, pages, depths, out)
PyObject *call_cache_step(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        need_args(n, 7);
        const at::Tensor &lens = device_tensor(args[0], "kv_lens");
        if (lens.scalar_type() != at::kInt || lens.dim() != 1 || !lens.is_contiguous()) fail("kv_lens must be contiguous int32 [B]");
        const at::Device device = lens.device();
        const int *counts = int_data(args[1], lens.sizes(), device, "counts must be contiguous int32 [B] on the device of kv_lens");
        const int S = as_int(args[2]), block_rows = as_int(args[3]);
        if (S < 0) return PyLong_FromLong(TSDPA_ERR_BAD_SHAPE);
        const int64_t B = lens.size(0);
        if (B * S > std::numeric_limits<int>::max()) return PyLong_FromLong(TSDPA_ERR_BAD_SHAPE);
        int *table = nullptr, *free_pages = nullptr;
        const int *pool = nullptr;
        int64_t max_blocks = 0, pool_size = 0;
        at::Tensor pages[3];                       // (a sequence that nobody else holds may be all that keeps them)
        if (args[4] != Py_None) {
            static const char text[] = "pages must be (block_table, free_pages, pool): contiguous int32 [B, max_blocks], [pool_size] and [2] on the device of kv_lens";
            each_of(args[4], 3, text, [&](Py_ssize_t i, PyObject *x) {
                if (!THPVariable_Check(x)) fail(text);
                const at::Tensor &t = pages[i] = THPVariable_Unpack(x);
                if (t.scalar_type() != at::kInt || t.device() != device || !t.is_contiguous() || t.dim() != (i == 0 ? 2 : 1)) fail(text);
                if (i == 0) {
                    if (t.size(0) != B) fail(text);
                    max_blocks = t.size(1);
                    table = (int *)data(t);
                } else if (i == 1) {
                    pool_size = t.size(0);
                    free_pages = (int *)data(t);
                } else {
                    if (t.size(0) != 2) fail(text);
                    pool = (const int *)data(t);
                }
            });
            const int64_t most = std::numeric_limits<int>::max();
            if (max_blocks > most || pool_size > most) return PyLong_FromLong(TSDPA_ERR_BAD_SHAPE);
            // (an empty tensor has no address: any that is not looked at says that there is a table)
            if (!table) table = (int *)pool;
            if (!free_pages) free_pages = (int *)pool;
        }
        const int *depths = nullptr;
        if (args[5] != Py_None) depths = int_data(args[5], {B, S}, device, "depths must be contiguous int32 [B, S] on the device of kv_lens");
        static const char text[] = "out must be (new_lens, slots, positions, new_pool): contiguous int32 [B], [B, S], [B, S] and [2] on the device of kv_lens";
        at::Tensor new_lens, slots, positions, new_pool;
        if (args[6] == Py_None) {
            Carver carve(2 * Carver::room(B * S, 4) + Carver::room(B, 4) + Carver::room(2, 4), lens);
            new_lens = carve.next(lens.sizes(), at::kInt);
            slots = carve.next({B, S}, at::kInt);
            positions = carve.next({B, S}, at::kInt);
            new_pool = carve.next({2}, at::kInt);
        } else {
            const Given<4> given(args[6], text);
            new_lens = made(given.t[0], lens.sizes(), at::kInt, lens, text);
            slots = made(given.t[1], {B, S}, at::kInt, lens, text);
            positions = made(given.t[2], {B, S}, at::kInt, lens, text);
            new_pool = made(given.t[3], {2}, at::kInt, lens, text);
            distinct({Extent(new_lens), Extent(slots), Extent(positions), Extent(new_pool)},
                     {Extent(lens), Extent(counts, B), Extent(depths, B * S), Extent(table, B * max_blocks), Extent(free_pages, pool_size), Extent(pool, 2)},
                     "new_lens, slots, positions and new_pool must be other tensors than each other and what the step reads (kv_lens and pool among it)");
        }
        if (B > std::numeric_limits<int>::max()) return PyLong_FromLong(TSDPA_ERR_BAD_SHAPE);
        const Launch on(lens);
        const int st = without_gil(tiled_sdpa_cache_step, (const int *)data(lens), counts, depths, table, free_pages, pool, (int *)data(new_lens), (int *)data(slots),
                                   (int *)data(positions), (int *)data(new_pool), (int)B, S, (int)max_blocks, block_rows, (int)pool_size, on.stream);
        return tuple_of(st, {&new_lens, &slots, &positions, &new_pool});
    });
}

// ---- norm and rotation of queries and keys

const at::Tensor &rows_tensor(PyObject *obj, const char *name)
{
    const at::Tensor &t = device_tensor(obj, name);
    if (t.dim() != 4 || (t.size(3) > 1 && t.stride(3) != 1)) fail_named(name, "must be [B, S, heads, D] with adjacent values in a row");
    return t;
}

tsdpa_rows rows_of(const at::Tensor &t) { return tsdpa_rows{data(t), (long long)t.stride(0), (long long)t.stride(1), (long long)t.stride(2)}; }

// What the three calls have in common: q, k, the weights, positions and frequencies, from the arguments that begin at args[0] (q, k,
// q_weight, k_weight, positions, inv_freq, axes, eps, interleaved).
struct Rope {
    tsdpa_rope p{};
    at::Tensor q, k;
    at::Tensor weight[2];
    int64_t n_positions = 0;
    explicit Rope(PyObject *const *args)
    {
        q = rows_tensor(args[0], "q");
        k = rows_tensor(args[1], "k");
        p.dtype = element_type(q);
        const at::IntArrayRef s = q.sizes(), t = k.sizes();
        if (k.scalar_type() != q.scalar_type() || k.device() != q.device() || t[0] != s[0] || t[1] != s[1] || t[3] != s[3])
            fail("q and k must be [B, S, H, D] and [B, S, Hkv, D] of one dtype and device");
        for (int i = 0; i < 4; ++i)
            if (s[i] > std::numeric_limits<int>::max() || t[i] > std::numeric_limits<int>::max()) fail("q and k are too large");
        p.B = (int)s[0];
        p.S = (int)s[1];
        p.H = (int)s[2];
        p.Hkv = (int)t[2];
        p.D = (int)s[3];
        p.weight_dtype = p.dtype;
        for (int i = 0; i < 2; ++i) {
            static const char text[] = "q_weight and k_weight must be contiguous [D] in float32 or the dtype of q, both the same, on the device of q (or None)";
            if (args[2 + i] == Py_None) continue;
            if (!THPVariable_Check(args[2 + i])) fail(text);
            const at::Tensor &w = THPVariable_Unpack(args[2 + i]);
            if (w.dim() != 1 || w.size(0) != s[3] || !w.is_contiguous() || w.device() != q.device() ||
                (w.scalar_type() != at::kFloat && w.scalar_type() != q.scalar_type()) ||
                (i == 1 && weight[0].defined() && w.scalar_type() != weight[0].scalar_type()))
                fail(text);
            weight[i] = w;
            if (w.scalar_type() == at::kFloat) p.weight_dtype = TSDPA_F32;
        }
        if (weight[0].defined()) p.q_weight = data(weight[0]);
        if (weight[1].defined()) p.k_weight = data(weight[1]);
        if (!THPVariable_Check(args[5])) fail("inv_freq must be contiguous float32 [rot / 2] on the device of q");
        const at::Tensor &f = THPVariable_Unpack(args[5]);
        if (f.scalar_type() != at::kFloat || f.dim() != 1 || !f.is_contiguous() || f.device() != q.device() || f.size(0) > s[3])
            fail("inv_freq must be contiguous float32 [rot / 2] on the device of q");
        p.rot = 2 * (int)f.size(0);
        p.inv_freq = (const float *)data(f);
        const bool several = args[6] != Py_None;
        {
            static const char text[] = "positions must be contiguous int32 [S] or [B, S] on the device of q, with axes [A, S] or [A, B, S]";
            if (!THPVariable_Check(args[4])) fail(text);
            const at::Tensor &x = THPVariable_Unpack(args[4]);
            const int64_t lead = several ? 1 : 0, dims = x.dim() - lead;
            if (x.scalar_type() != at::kInt || !x.is_contiguous() || x.device() != q.device() || (dims != 1 && dims != 2) ||
                x.size(x.dim() - 1) != s[1] || (dims == 2 && x.size(lead) != s[0]))
                fail(text);
            if (several && (x.size(0) < 1 || x.size(0) > std::numeric_limits<int>::max())) fail(text);
            p.positions = (const int *)data(x);
            n_positions = x.numel();
            p.pos_batch = dims == 2 ? (long long)s[1] : 0;
            p.pos_axis = dims == 2 ? (long long)(s[0] * s[1]) : (long long)s[1];
            p.n_axes = several ? (int)x.size(0) : 1;
        }
        if (several) p.axes = int_data(args[6], f.sizes(), q.device(), "axes must be contiguous int32 [rot / 2] on the device of q");
        const double eps = PyFloat_AsDouble(args[7]);
        if (eps == -1.0 && PyErr_Occurred()) throw PyFail{};
        p.eps = (float)eps;
        p.flags = as_bool(args[8]) ? (unsigned)TSDPA_FLAG_INTERLEAVED : 0u;
    }
    // Refuses outputs that overlap each other or what the kernel reads (`rows` and the arguments).
    void apart(std::initializer_list<Extent> outputs, std::initializer_list<Extent> rows, const char *complaint) const
    {
        distinct(outputs, rows, complaint);
        const int64_t weight_bytes = (int64_t)p.D * (p.weight_dtype == TSDPA_F32 ? 4 : 2), pairs = p.rot / 2;
        for (const Extent &i : {Extent(p.q_weight, weight_bytes), Extent(p.k_weight, weight_bytes), Extent(p.positions, n_positions),
                                Extent((const void *)p.inv_freq, pairs * (int64_t)sizeof(float)), Extent(p.axes, pairs)})
            for (const Extent &o : outputs)
                if (o.meets(i)) fail(complaint);
    }
    // [B, heads, S, D], as attention reads them
    at::Tensor heads_out(const at::Tensor &given, const at::Tensor &x, const char *complaint) const
    {
        return made(given, {x.size(0), x.size(2), x.size(1), x.size(3)}, q.scalar_type(), q, complaint);
    }
};

// qk_norm_rope(q, k, q_weight, k_weight, positions, inv_freq, axes, eps, interleaved, out)
PyObject *call_qk_norm_rope(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        need_args(n, 10);
        const Rope r(args);
        static const char text[] = "out must be (q_out, k_out): contiguous [B, H, S, D] and [B, Hkv, S, D] like q and k";
        const Given<2> given(args[9], text);
        const at::Tensor q_out = r.heads_out(given.t[0], r.q, text), k_out = r.heads_out(given.t[1], r.k, text);
        if (args[9] != Py_None) r.apart({Extent(q_out), Extent(k_out)}, {Extent(r.q), Extent(r.k)}, "q_out and k_out must overlap neither each other nor what the call reads");
        const tsdpa_rows q = rows_of(r.q), k = rows_of(r.k);
        const Launch on(r.q);
        const int st = without_gil(tiled_sdpa_qk_norm_rope, &r.p, &q, &k, data(q_out), data(k_out), on.stream);
        return tuple_of(st, {&q_out, &k_out});
    });
}

// qk_norm_rope_cache(q, k, q_weight, k_weight, positions, inv_freq, axes, eps, interleaved, v, k_cache, v_cache, slots, out)
PyObject *call_qk_norm_rope_cache(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        need_args(n, 14);
        const Rope r(args);
        const at::Tensor &v = rows_tensor(args[9], "v"), &kc = heads_tensor(args[10], "k_cache"), &vc = heads_tensor(args[11], "v_cache");
        if (!same_sizes(v, r.k) || v.scalar_type() != r.k.scalar_type() || v.device() != r.k.device()) fail("v must match k in shape, dtype and device");
        const at::IntArrayRef c = kc.sizes();
        if (!same_sizes(kc, vc) || kc.scalar_type() != r.q.scalar_type() || vc.scalar_type() != r.q.scalar_type() || kc.device() != r.q.device() ||
            vc.device() != r.q.device() || c[1] != r.p.Hkv || c[3] != r.p.D)
            fail("k_cache, v_cache must be [pages, Hkv, block_rows, D] of the dtype and device of q");
        if (c[0] > std::numeric_limits<int>::max() || c[2] > std::numeric_limits<int>::max()) return PyLong_FromLong(TSDPA_ERR_BAD_SHAPE);
        const int *slots = int_data(args[12], r.q.sizes().slice(0, 2), r.q.device(), "slots must be contiguous int32 [B, S] on the device of q");
        static const char text[] = "out must be contiguous [B, H, S, D] like q";
        if (args[13] != Py_None && !THPVariable_Check(args[13])) fail(text);
        const at::Tensor q_out = r.heads_out(args[13] == Py_None ? at::Tensor() : THPVariable_Unpack(args[13]), r.q, text);
        r.apart({Extent(kc), Extent(vc), args[13] == Py_None ? Extent() : Extent(q_out)},      // (a new tensor overlaps nothing)
                {Extent(r.q), Extent(r.k), Extent(v), Extent(slots, (int64_t)r.p.B * r.p.S)},
                "the result, k_cache and v_cache must overlap neither each other nor what the call reads");
        const tsdpa_rows q = rows_of(r.q), k = rows_of(r.k), vr = rows_of(v);
        const Launch on(r.q);
        const int st = without_gil(tiled_sdpa_qk_norm_rope_cache, &r.p, &q, &k, &vr, slots, data(q_out), data(kc), data(vc), (int)c[0], (int)c[2], on.stream);
        if (st != TSDPA_OK) return PyLong_FromLong(st);
        return give(args[13], q_out);
    });
}

// qk_norm_rope_backward(q, k, q_weight, k_weight, positions, inv_freq, axes, eps, interleaved, dq_out, dk_out, workspace, grads)
PyObject *call_qk_norm_rope_backward(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        need_args(n, 13);
        const Rope r(args);
        const at::Tensor &dq_out = heads_tensor(args[9], "dq_out"), &dk_out = heads_tensor(args[10], "dk_out");
        auto agree = [&](const at::Tensor &g, const at::Tensor &x) {
            const int64_t shape[4] = {x.size(0), x.size(2), x.size(1), x.size(3)};
            if (g.sizes() != at::IntArrayRef(shape, 4) || g.scalar_type() != x.scalar_type() || g.device() != x.device())
                fail("dq_out and dk_out must be [B, H, S, D] and [B, Hkv, S, D] of the dtype and device of q and k");
        };
        agree(dq_out, r.q);
        agree(dk_out, r.k);
        at::Tensor dx[2], dw[2];
        if (args[12] == Py_None) {
            dx[0] = empty(r.q.sizes(), r.q.scalar_type(), r.q);
            dx[1] = empty(r.k.sizes(), r.q.scalar_type(), r.q);
        } else {
            static const char text[] = "grads must be (dq, dk): [B, S, heads, D] like q and k, with adjacent values in a row";
            const Given<2> given(args[12], text);
            for (int i = 0; i < 2; ++i) {
                const at::Tensor &t = given.t[i], &like = i == 0 ? r.q : r.k;
                if (!same_sizes(t, like) || t.scalar_type() != like.scalar_type() || t.device() != like.device() || (t.size(3) > 1 && t.stride(3) != 1)) fail(text);
                dx[i] = t;
            }
            // (of q and k the norm's rows are read, no others)
            const auto read = [&](int i, const at::Tensor &x) { return r.weight[i].defined() ? Extent(x) : Extent(); };
            r.apart({Extent(dx[0]), Extent(dx[1])}, {Extent(dq_out), Extent(dk_out), read(0, r.q), read(1, r.k)}, "dq and dk must overlap neither each other nor what the call reads");
        }
        for (int i = 0; i < 2; ++i)
            if (r.weight[i].defined()) dw[i] = empty(r.weight[i].sizes(), r.weight[i].scalar_type(), r.q);
        const bool norms = dw[0].defined() || dw[1].defined();
        const Workspace ws(args[11], norms ? tiled_sdpa_qk_norm_rope_bwd_workspace_bytes(r.p.B, r.p.S, r.p.D) : 0, r.q);
        const tsdpa_rows q = rows_of(r.q), k = rows_of(r.k), dq = rows_of(dx[0]), dk = rows_of(dx[1]);
        const Launch on(r.q);
        const int st = without_gil(tiled_sdpa_qk_norm_rope_bwd, &r.p, (const void *)data(dq_out), (const void *)data(dk_out), &q, &k, &dq, &dk,
                                   dw[0].defined() ? data(dw[0]) : nullptr, dw[1].defined() ? data(dw[1]) : nullptr, ws.ptr, ws.bytes, on.stream);
        return tuple_of(st, {&dx[0], &dx[1], &dw[0], &dw[1]});
    });
}

PyMethodDef methods[] = {
    {"sdpa", (PyCFunction)(void (*)(void))call_sdpa, METH_FASTCALL, nullptr},
    {"sdpa_kv", (PyCFunction)(void (*)(void))call_sdpa_kv, METH_FASTCALL, nullptr},
    {"sdpa_paged", (PyCFunction)(void (*)(void))call_sdpa_paged, METH_FASTCALL, nullptr},
    {"sdpa_backward", (PyCFunction)(void (*)(void))call_sdpa_backward, METH_FASTCALL, nullptr},
    {"sdpa_tree", (PyCFunction)(void (*)(void))call_sdpa_tree, METH_FASTCALL, nullptr},
    {"tree_mask", (PyCFunction)(void (*)(void))call_tree_mask, METH_FASTCALL, nullptr},
    {"cache_step", (PyCFunction)(void (*)(void))call_cache_step, METH_FASTCALL, nullptr},
    {"qk_norm_rope", (PyCFunction)(void (*)(void))call_qk_norm_rope, METH_FASTCALL, nullptr},
    {"qk_norm_rope_cache", (PyCFunction)(void (*)(void))call_qk_norm_rope_cache, METH_FASTCALL, nullptr},
    {"qk_norm_rope_backward", (PyCFunction)(void (*)(void))call_qk_norm_rope_backward, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_calls", "tensor entry points of tiled SDPA", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls(void) { return PyModule_Create(&module); }
