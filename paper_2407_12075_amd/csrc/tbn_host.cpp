// Native form of the binding's everyday calls (module paper_2407_12075_amd._tbn_host).
//
// A call through ctypes costs the host 9 - 11 us (reading a dozen tensor attributes, allocating the output, looking up
// the stream, marshalling), more than the small kernels take.  Here the same checks, allocations and library calls are made on
// the C++ tensors.  Only the plain form of a call is taken: exact torch tensors that pass every check, integer arguments,
// outputs and workspaces left to the call, the current stream, no dispatch or function mode.  Anything else returns None and nothing has
// happened: the Python wrapper then runs its own code, which also words every error.
// One token through a 4096 x 4096 bfloat16 layer, calls in a row: 11.3 us through ctypes, 4.2 here (the kernel takes 3.5).
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <pybind11/pybind11.h>
#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>

#include "../../include/tbn.h"

namespace {

PyObject *g_raise = nullptr;   // the binding's _raise(status)

// The library is loaded by the binding; its entry points are handed over as addresses so that there is one instance.
decltype(&tbn_pack_workspace_bytes) p_pack_workspace_bytes;
decltype(&tbn_pack_tile) p_pack_tile;
decltype(&tbn_linear_forward) p_linear_forward;
decltype(&tbn_conv2d_forward) p_conv2d_forward;
decltype(&tbn_linear_coltiled_workspace_bytes) p_coltiled_workspace_bytes;
decltype(&tbn_linear_coltiled_forward) p_coltiled_forward;
decltype(&tbn_sign_pack) p_sign_pack;
decltype(&tbn_linear_forward_binact) p_forward_binact;
decltype(&tbn_kv_reserve) p_kv_reserve;
decltype(&tbn_kv_workspace_bytes) p_kv_workspace_bytes;
decltype(&tbn_kv_fork) p_kv_fork;
decltype(&tbn_kv_release) p_kv_release;
decltype(&tbn_kv_copy_pages) p_kv_copy_pages;
decltype(&tbn_kv_append) p_kv_append;
decltype(&tbn_kv_keep) p_kv_keep;
decltype(&tbn_tree_attention_workspace_bytes) p_tree_attention_workspace_bytes;
decltype(&tbn_tree_attention) p_tree_attention;
decltype(&tbn_window_attention_workspace_bytes) p_window_attention_workspace_bytes;
decltype(&tbn_window_attention) p_window_attention;
decltype(&tbn_kv4_append) p_kv4_append;
decltype(&tbn_kv4_read) p_kv4_read;
decltype(&tbn_kv4_copy_pages) p_kv4_copy_pages;
decltype(&tbn_kv4_keep) p_kv4_keep;
decltype(&tbn_kv4_attention_workspace_bytes) p_kv4_attention_workspace_bytes;
decltype(&tbn_kv4_attention) p_kv4_attention;
decltype(&tbn_verify_workspace_bytes) p_verify_workspace_bytes;
decltype(&tbn_verify) p_verify;
decltype(&tbn_block_select_workspace_bytes) p_block_select_workspace_bytes;
decltype(&tbn_block_select) p_block_select;
decltype(&tbn_block_attention_workspace_bytes) p_block_attention_workspace_bytes;
decltype(&tbn_block_attention) p_block_attention;

constexpr int64_t kMaxElems = int64_t(1) << 40;

// a plain dense tensor on a GPU
const at::Tensor *plain(PyObject *o, int64_t dims = -1) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || (dims >= 0 && t.dim() != dims) || !t.is_contiguous()) return nullptr;
    constexpr c10::DispatchKeySet kWrapped({c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
                                            c10::DispatchKey::Functionalize, c10::DispatchKey::Python});
    if (t.key_set().has_any(kWrapped)) return nullptr;
    return &t;
}

const at::Tensor *plain(PyObject *o, at::ScalarType st, const at::Tensor &with) {
    const at::Tensor *t = plain(o);
    return t && t->scalar_type() == st && t->device() == with.device() ? t : nullptr;
}

bool activations(const at::Tensor &x, tbn_dtype &dt) {
    if (x.scalar_type() == at::kBFloat16) dt = TBN_BF16;
    else if (x.scalar_type() == at::kFloat) dt = TBN_F32;
    else return false;
    return true;
}

bool ordinary_context() {
    return !c10::impl::dispatch_mode_enabled() && !at::impl::torch_function_mode_enabled() &&
           !c10::impl::tls_local_dispatch_key_set().included_.has(c10::DispatchKey::FuncTorchDynamicLayerFrontMode);
}

bool integer(PyObject *o, int64_t lo, int64_t hi, int64_t &v) {
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return overflow == 0 && v >= lo && v <= hi;
}

bool pair(PyObject *o, int64_t lo, int64_t hi, int64_t &a, int64_t &b) {
    return PyTuple_CheckExact(o) && PyTuple_GET_SIZE(o) == 2 && integer(PyTuple_GET_ITEM(o, 0), lo, hi, a) &&
           integer(PyTuple_GET_ITEM(o, 1), lo, hi, b);
}

// n weights, n % k == 0 and a tile and alphas that hold them: what the library cannot see behind raw pointers
bool layer(int64_t rows, int64_t row_len, int64_t k, const at::Tensor &tile, const at::Tensor &alpha) {
    int64_t n;
    if (__builtin_mul_overflow(rows, row_len, &n) || n > kMaxElems || n % k != 0) return false;
    return tile.numel() >= (n / k + 31) / 32 && alpha.numel() >= 1 && alpha.numel() <= INT32_MAX;
}

void *stream() { return c10::hip::getCurrentHIPStream().stream(); }

uint32_t *words(const at::Tensor &t) { return static_cast<uint32_t *>(t.data_ptr()); }
float *floats(const at::Tensor &t) { return static_cast<float *>(t.data_ptr()); }

// the wrapper's result, or the binding's exception for this status
PyObject *result(tbn_status st, PyObject *(*make)(const at::Tensor &, const at::Tensor &), const at::Tensor &a, const at::Tensor &b) {
    if (st == TBN_OK) return make(a, b);
    PyObject *r = PyObject_CallFunction(g_raise, "i", static_cast<int>(st));
    Py_XDECREF(r);
    return nullptr;
}
PyObject *one(const at::Tensor &a, const at::Tensor &) { return THPVariable_Wrap(a); }
PyObject *two(const at::Tensor &a, const at::Tensor &b) {
    PyObject *pa = THPVariable_Wrap(a), *pb = THPVariable_Wrap(b);
    PyObject *r = pa && pb ? PyTuple_Pack(2, pa, pb) : nullptr;
    Py_XDECREF(pa);
    Py_XDECREF(pb);
    return r;
}

// (x, tile, alpha, out_features, k, flags)
PyObject *linear_forward(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    int64_t out, k, flags;
    tbn_dtype dt;
    if (n_args != 6 || !ordinary_context()) Py_RETURN_NONE;
    const at::Tensor *x = plain(args[0], 2);
    if (!x || !activations(*x, dt)) Py_RETURN_NONE;
    const at::Tensor *tile = plain(args[1], at::kInt, *x), *alpha = plain(args[2], at::kFloat, *x);
    if (!tile || !alpha || !integer(args[3], 1, kMaxElems, out) || !integer(args[4], 1, INT32_MAX, k) ||
        !integer(args[5], 0, UINT32_MAX, flags) || !layer(out, x->size(1), k, *tile, *alpha))
        Py_RETURN_NONE;
    const int64_t M = x->size(0), in = x->size(1);
    at::Tensor y = at::empty({M, out}, x->options());
    tbn_status st;
    {
        pybind11::gil_scoped_release no_gil;
        st = p_linear_forward(x->data_ptr(), y.data_ptr(), dt, M, in, out, words(*tile), static_cast<int32_t>(k), floats(*alpha),
                              static_cast<int32_t>(alpha->numel()), static_cast<uint32_t>(flags), stream());
    }
    return result(st, one, y, y);
    END_HANDLE_TH_ERRORS
}

// (x, tile, alpha, out_channels, kh, kw, k, stride, pad, flags)
PyObject *conv2d_forward(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    int64_t O, kh, kw, k, sh, sw, ph, pw, flags;
    tbn_dtype dt;
    constexpr int64_t kSmall = 1 << 20;
    if (n_args != 10 || !ordinary_context()) Py_RETURN_NONE;
    const at::Tensor *x = plain(args[0], 4);
    if (!x || !activations(*x, dt)) Py_RETURN_NONE;
    const at::Tensor *tile = plain(args[1], at::kInt, *x), *alpha = plain(args[2], at::kFloat, *x);
    if (!tile || !alpha || !integer(args[3], 1, 1 << 24, O) || !integer(args[4], 1, 4096, kh) || !integer(args[5], 1, 4096, kw) ||
        !integer(args[6], 1, INT32_MAX, k) || !pair(args[7], 1, kSmall, sh, sw) || !pair(args[8], 0, kSmall, ph, pw) ||
        !integer(args[9], 0, UINT32_MAX, flags))
        Py_RETURN_NONE;
    const int64_t N = x->size(0), C = x->size(1), H = x->size(2), W = x->size(3);
    if (C > (1 << 24) || H + 2 * ph < kh || W + 2 * pw < kw || !layer(O, C * kh * kw, k, *tile, *alpha)) Py_RETURN_NONE;
    at::Tensor y = at::empty({N, O, (H + 2 * ph - kh) / sh + 1, (W + 2 * pw - kw) / sw + 1}, x->options());
    tbn_status st;
    {
        pybind11::gil_scoped_release no_gil;
        st = p_conv2d_forward(x->data_ptr(), y.data_ptr(), dt, N, C, H, W, O, static_cast<int32_t>(kh), static_cast<int32_t>(kw),
                              static_cast<int32_t>(sh), static_cast<int32_t>(sw), static_cast<int32_t>(ph), static_cast<int32_t>(pw),
                              words(*tile), static_cast<int32_t>(k), floats(*alpha), static_cast<int32_t>(alpha->numel()),
                              static_cast<uint32_t>(flags), stream());
    }
    return result(st, one, y, y);
    END_HANDLE_TH_ERRORS
}

// (x, tile, alpha, out_features, k, flags); the workspace is the call's own
PyObject *linear_coltiled_forward(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    int64_t out, k, flags;
    tbn_dtype dt;
    if (n_args != 6 || !ordinary_context()) Py_RETURN_NONE;
    const at::Tensor *x = plain(args[0], 2);
    if (!x || !activations(*x, dt)) Py_RETURN_NONE;
    const at::Tensor *tile = plain(args[1], at::kInt, *x), *alpha = plain(args[2], at::kFloat, *x);
    if (!tile || !alpha || !integer(args[3], 1, kMaxElems, out) || !integer(args[4], 1, INT32_MAX, k) ||
        !integer(args[5], 0, UINT32_MAX, flags) || !layer(out, x->size(1), k, *tile, *alpha))
        Py_RETURN_NONE;
    const int64_t M = x->size(0), in = x->size(1);
    const size_t need = std::max<size_t>(p_coltiled_workspace_bytes(dt, M, in, static_cast<int32_t>(k)), 16);
    at::Tensor y = at::empty({M, out}, x->options());
    at::Tensor ws = at::empty({static_cast<int64_t>(need)}, x->options().dtype(at::kByte));
    tbn_status st;
    {
        pybind11::gil_scoped_release no_gil;
        st = p_coltiled_forward(x->data_ptr(), y.data_ptr(), dt, M, in, out, words(*tile), static_cast<int32_t>(k), floats(*alpha),
                                static_cast<int32_t>(alpha->numel()), static_cast<uint32_t>(flags), ws.data_ptr(), need, stream());
    }
    return result(st, one, y, y);
    END_HANDLE_TH_ERRORS
}

// (x)
PyObject *sign_pack(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    tbn_dtype dt;
    if (n_args != 1 || !ordinary_context()) Py_RETURN_NONE;
    const at::Tensor *x = plain(args[0], 2);
    if (!x || !activations(*x, dt) || x->size(1) < 1) Py_RETURN_NONE;
    const int64_t M = x->size(0), in = x->size(1);
    at::Tensor bits = at::empty({M, (in + 31) / 32}, x->options().dtype(at::kInt));
    tbn_status st;
    {
        pybind11::gil_scoped_release no_gil;
        st = p_sign_pack(x->data_ptr(), dt, M, in, words(bits), stream());
    }
    return result(st, one, bits, bits);
    END_HANDLE_TH_ERRORS
}

// (xbits, in, tile, alpha, out_features, k, output is bfloat16, flags)
PyObject *linear_forward_binact(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    int64_t in, out, k, flags;
    if (n_args != 8 || !ordinary_context()) Py_RETURN_NONE;
    const at::Tensor *bits = plain(args[0], 2);
    if (!bits || bits->scalar_type() != at::kInt || !integer(args[1], 1, kMaxElems, in) || bits->size(1) != (in + 31) / 32)
        Py_RETURN_NONE;
    const at::Tensor *tile = plain(args[2], at::kInt, *bits), *alpha = plain(args[3], at::kFloat, *bits);
    if (!tile || !alpha || !integer(args[4], 1, kMaxElems, out) || !integer(args[5], 1, INT32_MAX, k) ||
        !integer(args[7], 0, UINT32_MAX, flags) || !layer(out, in, k, *tile, *alpha))
        Py_RETURN_NONE;
    const int64_t M = bits->size(0);
    const bool signs = (flags & TBN_FLAG_SIGN_OUT) != 0, bf16 = args[6] == Py_True;
    at::Tensor y = signs ? at::empty({M, (out + 31) / 32}, bits->options())
                         : at::empty({M, out}, bits->options().dtype(bf16 ? at::kBFloat16 : at::kFloat));
    tbn_status st;
    {
        pybind11::gil_scoped_release no_gil;
        st = p_forward_binact(words(*bits), y.data_ptr(), !signs && bf16 ? TBN_BF16 : TBN_F32, M, in, out, words(*tile),
                              static_cast<int32_t>(k), floats(*alpha), static_cast<int32_t>(alpha->numel()), static_cast<uint32_t>(flags),
                              stream());
    }
    return result(st, one, y, y);
    END_HANDLE_TH_ERRORS
}

// (w_real, k, n_alpha); the magnitudes are those of w_real, the outputs and the workspace the call's own
PyObject *pack_tile(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    int64_t k, n_alpha;
    if (n_args != 3 || !ordinary_context()) Py_RETURN_NONE;
    const at::Tensor *w = plain(args[0]);
    if (!w || w->scalar_type() != at::kFloat || !integer(args[1], 1, INT32_MAX, k) || !integer(args[2], 1, INT32_MAX, n_alpha))
        Py_RETURN_NONE;
    const int64_t n = w->numel();
    if (n < 1 || n % k != 0 || (n_alpha != 1 && n_alpha != k)) Py_RETURN_NONE;
    at::Tensor tile = at::empty({(n / k + 31) / 32}, w->options().dtype(at::kInt));
    at::Tensor alpha = at::empty({n_alpha}, w->options());
    const size_t need = std::max<size_t>(p_pack_workspace_bytes(n, static_cast<int32_t>(k), static_cast<int32_t>(n_alpha)), 8);
    at::Tensor ws = at::empty({static_cast<int64_t>(need)}, w->options().dtype(at::kByte));
    tbn_status st;
    {
        pybind11::gil_scoped_release no_gil;
        st = p_pack_tile(floats(*w), nullptr, n, static_cast<int32_t>(k), static_cast<int32_t>(n_alpha), words(tile), floats(alpha),
                         ws.data_ptr(), need, stream());
    }
    return result(st, two, tile, alpha);
    END_HANDLE_TH_ERRORS
}

// ---- the paged cache ------------------------------------------------------------------------------------------------------
// Pools and indices come as (address of the C struct, GPU): the Python object that holds the struct checked its tensors once.

struct Held {
    const void *at;
    int64_t gpu;
};

bool held(PyObject *address, PyObject *gpu, Held &h) {
    if (!PyLong_CheckExact(address) || !integer(gpu, 0, 1 << 20, h.gpu)) return false;
    h.at = PyLong_AsVoidPtr(address);
    if (PyErr_Occurred()) PyErr_Clear();
    return h.at != nullptr;
}

const tbn_kv_pool *pool_of(const Held &h) { return static_cast<const tbn_kv_pool *>(h.at); }
const tbn_kv4_pool *pool4_of(const Held &h) { return static_cast<const tbn_kv4_pool *>(h.at); }
const tbn_kv_index *index_of(const Held &h) { return static_cast<const tbn_kv_index *>(h.at); }

// a dense int32 tensor of at least n entries on the GPU
int32_t *ints(PyObject *o, int64_t n, int64_t gpu) {
    const at::Tensor *t = plain(o);
    if (!t || t->scalar_type() != at::kInt || t->numel() < n || t->device().index() != gpu) return nullptr;
    return static_cast<int32_t *>(t->data_ptr());
}

// (tokens, heads, dim) of type dt, heads dense, tokens `stride` elements apart (heads 0: any number)
const at::Tensor *rows_of(PyObject *o, int64_t gpu, int64_t dim, at::ScalarType dt, int64_t heads, int64_t &stride) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    constexpr c10::DispatchKeySet kWrapped({c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
                                            c10::DispatchKey::Functionalize, c10::DispatchKey::Python});
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.dim() != 3 || t.key_set().has_any(kWrapped)) return nullptr;
    if (t.device().index() != gpu || t.scalar_type() != dt) return nullptr;
    const int64_t n = t.size(0), h = t.size(1), d = t.size(2);
    if (d != dim || h < 1 || h > 65536 || (heads && h != heads) || n < 1) return nullptr;
    if (t.stride(2) != 1 || (h > 1 && t.stride(1) != d) || (n > 1 && t.stride(0) < h * d)) return nullptr;
    stride = n > 1 ? t.stride(0) : h * d;
    return &t;
}
// of the pool's type
const at::Tensor *rows(PyObject *o, const Held &pool, int64_t heads, int64_t &stride) {
    return rows_of(o, pool.gpu, pool_of(pool)->dim, pool_of(pool)->dt == TBN_F32 ? at::kFloat : at::kBFloat16, heads, stride);
}
// for a pool in 4 bits: of either type
const at::Tensor *rows4(PyObject *o, const Held &pool, int64_t heads, int64_t &stride, tbn_dtype &dt) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.defined() && activations(t, dt) ? rows_of(o, pool.gpu, pool4_of(pool)->dim, t.scalar_type(), heads, stride) : nullptr;
}

// the library's call, without the interpreter's lock: a launch may wait for room in a queue
template <typename Call>
tbn_status unlocked(Call call) {
    pybind11::gil_scoped_release no_gil;
    return call();
}

PyObject *none(tbn_status st) {
    if (st == TBN_OK) Py_RETURN_TRUE;   // done, nothing to return (None would be "not taken")
    PyObject *r = PyObject_CallFunction(g_raise, "i", static_cast<int>(st));
    Py_XDECREF(r);
    return nullptr;
}

at::Tensor bytes_like(const at::Tensor &t, size_t n) { return at::empty({static_cast<int64_t>(n)}, t.options().dtype(at::kByte)); }

// (index, gpu, n_new)
PyObject *kv_reserve(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    Held ix;
    if (n_args != 3 || !ordinary_context() || !held(args[0], args[1], ix)) Py_RETURN_NONE;
    const int64_t n = index_of(ix)->n_seqs;
    const int32_t *fresh = ints(args[2], n, ix.gpu);
    if (!fresh) Py_RETURN_NONE;
    const at::Tensor &like = THPVariable_Unpack(args[2]);
    at::Tensor src = at::empty({n}, like.options()), dst = at::empty({n}, like.options());
    const size_t need = p_kv_workspace_bytes(index_of(ix)->n_pages, static_cast<int32_t>(n));
    at::Tensor ws = bytes_like(like, need);
    const tbn_status st = unlocked([&] {
        return p_kv_reserve(index_of(ix), fresh, static_cast<int32_t *>(src.data_ptr()), static_cast<int32_t *>(dst.data_ptr()), ws.data_ptr(), need, stream());
    });
    return result(st, two, src, dst);
    END_HANDLE_TH_ERRORS
}

// (index, gpu, parents, children)
PyObject *kv_fork(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    Held ix;
    if (n_args != 4 || !ordinary_context() || !held(args[0], args[1], ix)) Py_RETURN_NONE;
    const int32_t *a = ints(args[2], 0, ix.gpu), *b = ints(args[3], 0, ix.gpu);
    if (!a || !b) Py_RETURN_NONE;
    const int64_t n = THPVariable_Unpack(args[2]).numel();
    if (THPVariable_Unpack(args[3]).numel() != n || n > INT32_MAX) Py_RETURN_NONE;
    return none(unlocked([&] { return p_kv_fork(index_of(ix), a, b, static_cast<int32_t>(n), stream()); }));
    END_HANDLE_TH_ERRORS
}

// (index, gpu, keep)
PyObject *kv_release(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    Held ix;
    if (n_args != 3 || !ordinary_context() || !held(args[0], args[1], ix)) Py_RETURN_NONE;
    const int32_t *keep = ints(args[2], index_of(ix)->n_seqs, ix.gpu);
    if (!keep) Py_RETURN_NONE;
    return none(unlocked([&] { return p_kv_release(index_of(ix), keep, stream()); }));
    END_HANDLE_TH_ERRORS
}

// (pool, gpu, src, dst, count or None)
template <typename Call>
PyObject *copy_pages(PyObject *const *args, Py_ssize_t n_args, Call call) {
    Held pool;
    if (n_args != 5 || !ordinary_context() || !held(args[0], args[1], pool)) Py_RETURN_NONE;
    const int32_t *a = ints(args[2], 0, pool.gpu), *b = ints(args[3], 0, pool.gpu), *count = args[4] == Py_None ? nullptr : ints(args[4], 1, pool.gpu);
    if (!a || !b || (!count && args[4] != Py_None)) Py_RETURN_NONE;
    const int64_t n = THPVariable_Unpack(args[2]).numel();
    if (THPVariable_Unpack(args[3]).numel() != n) Py_RETURN_NONE;
    return none(unlocked([&] { return call(pool, a, b, n, count); }));
}
PyObject *kv_copy_pages(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    return copy_pages(args, n_args, [](const Held &pool, const int32_t *a, const int32_t *b, int64_t n, const int32_t *count) {
        return p_kv_copy_pages(pool_of(pool), a, b, n, count, stream());
    });
    END_HANDLE_TH_ERRORS
}
PyObject *kv4_copy_pages(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    if (!p_kv4_copy_pages) Py_RETURN_NONE;
    return copy_pages(args, n_args, [](const Held &pool, const int32_t *a, const int32_t *b, int64_t n, const int32_t *count) {
        return p_kv4_copy_pages(pool4_of(pool), a, b, n, count, stream());
    });
    END_HANDLE_TH_ERRORS
}

// (pool, gpu, index, gpu, k_new, v_new, cu_new, max_new)
PyObject *kv_append(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    Held pool, ix;
    int64_t most, ks, vs;
    if (n_args != 8 || !ordinary_context() || !held(args[0], args[1], pool) || !held(args[2], args[3], ix) || pool.gpu != ix.gpu) Py_RETURN_NONE;
    const at::Tensor *k = rows(args[4], pool, pool_of(pool)->kv_heads, ks), *v = rows(args[5], pool, pool_of(pool)->kv_heads, vs);
    const int32_t *cu = ints(args[6], int64_t(index_of(ix)->n_seqs) + 1, ix.gpu);
    if (!k || !v || !cu || k->size(0) != v->size(0) || !integer(args[7], 0, INT32_MAX, most)) Py_RETURN_NONE;
    return none(unlocked([&] { return p_kv_append(pool_of(pool), index_of(ix), k->data_ptr(), ks, v->data_ptr(), vs, cu, k->size(0), static_cast<int32_t>(most), stream()); }));
    END_HANDLE_TH_ERRORS
}

// (pool, gpu, index, gpu, k_new, v_new, cu_new, max_new)
PyObject *kv4_append(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    Held pool, ix;
    int64_t most, ks, vs;
    tbn_dtype dt, vt;
    if (!p_kv4_append || n_args != 8 || !ordinary_context() || !held(args[0], args[1], pool) || !held(args[2], args[3], ix) || pool.gpu != ix.gpu) Py_RETURN_NONE;
    const at::Tensor *k = rows4(args[4], pool, pool4_of(pool)->kv_heads, ks, dt), *v = rows4(args[5], pool, pool4_of(pool)->kv_heads, vs, vt);
    const int32_t *cu = ints(args[6], int64_t(index_of(ix)->n_seqs) + 1, ix.gpu);
    if (!k || !v || !cu || dt != vt || k->size(0) != v->size(0) || !integer(args[7], 0, INT32_MAX, most)) Py_RETURN_NONE;
    return none(unlocked([&] { return p_kv4_append(pool4_of(pool), index_of(ix), k->data_ptr(), ks, v->data_ptr(), vs, dt, cu, k->size(0), static_cast<int32_t>(most), stream()); }));
    END_HANDLE_TH_ERRORS
}

// (pool, gpu, index, gpu, cu, max_n, total, float32)
PyObject *kv4_read(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    Held pool, ix;
    int64_t most, total;
    if (!p_kv4_read || n_args != 8 || !ordinary_context() || !held(args[0], args[1], pool) || !held(args[2], args[3], ix) || pool.gpu != ix.gpu) Py_RETURN_NONE;
    const int32_t *cu = ints(args[4], int64_t(index_of(ix)->n_seqs) + 1, ix.gpu);
    if (!cu || !integer(args[5], 0, INT32_MAX, most) || !integer(args[6], 1, 1 << 30, total) || !PyBool_Check(args[7])) Py_RETURN_NONE;
    const bool f32 = args[7] == Py_True;
    const auto *p = pool4_of(pool);
    const auto options = THPVariable_Unpack(args[4]).options().dtype(f32 ? at::kFloat : at::kBFloat16);
    at::Tensor k = at::empty({total, p->kv_heads, p->dim}, options), v = at::empty({total, p->kv_heads, p->dim}, options);
    const tbn_status st = unlocked([&] {
        return p_kv4_read(p, index_of(ix), k.data_ptr(), v.data_ptr(), f32 ? TBN_F32 : TBN_BF16, cu, total, static_cast<int32_t>(most), stream());
    });
    return result(st, two, k, v);
    END_HANDLE_TH_ERRORS
}

// (pool, gpu, index, gpu, base, picks, counts)
template <typename Call>
PyObject *keep_keys(PyObject *const *args, Py_ssize_t n_args, Call call) {
    Held pool, ix;
    if (n_args != 7 || !ordinary_context() || !held(args[0], args[1], pool) || !held(args[2], args[3], ix) || pool.gpu != ix.gpu) Py_RETURN_NONE;
    const int64_t n = index_of(ix)->n_seqs;
    const int32_t *base = ints(args[4], n, ix.gpu), *picks = ints(args[5], 0, ix.gpu), *counts = ints(args[6], n, ix.gpu);
    if (!base || !picks || !counts) Py_RETURN_NONE;
    const at::Tensor &t = THPVariable_Unpack(args[5]);
    if (t.dim() != 2 || t.size(0) != n || t.size(1) > INT32_MAX) Py_RETURN_NONE;
    return none(unlocked([&] { return call(pool, index_of(ix), base, picks, static_cast<int32_t>(t.size(1)), counts); }));
}
PyObject *kv_keep(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    return keep_keys(args, n_args, [](const Held &pool, const tbn_kv_index *ix, const int32_t *base, const int32_t *picks, int32_t width, const int32_t *counts) {
        return p_kv_keep(pool_of(pool), ix, base, picks, width, counts, stream());
    });
    END_HANDLE_TH_ERRORS
}
PyObject *kv4_keep(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    if (!p_kv4_keep) Py_RETURN_NONE;
    return keep_keys(args, n_args, [](const Held &pool, const tbn_kv_index *ix, const int32_t *base, const int32_t *picks, int32_t width, const int32_t *counts) {
        return p_kv4_keep(pool4_of(pool), ix, base, picks, width, counts, stream());
    });
    END_HANDLE_TH_ERRORS
}

struct QueryArgs {
    Held pool, ix;
    const at::Tensor *q;
    int64_t stride, max_q, max_len;
    const int32_t *cu;
    tbn_dtype dt;
};

// (q, pool, gpu, index, gpu, cu_q, max_q, max_len or None, ...)
bool queries(PyObject *const *args, QueryArgs &a, bool four = false) {
    if (!ordinary_context() || !held(args[1], args[2], a.pool) || !held(args[3], args[4], a.ix) || a.pool.gpu != a.ix.gpu) return false;
    a.q = four ? rows4(args[0], a.pool, 0, a.stride, a.dt) : rows(args[0], a.pool, 0, a.stride);
    if (!a.q || a.q->size(1) % (four ? pool4_of(a.pool)->kv_heads : pool_of(a.pool)->kv_heads)) return false;
    a.cu = ints(args[5], int64_t(index_of(a.ix)->n_seqs) + 1, a.ix.gpu);
    a.max_len = 0;
    return a.cu && integer(args[6], 0, INT32_MAX, a.max_q) && (args[7] == Py_None || integer(args[7], 0, kMaxElems, a.max_len));
}

bool scale_of(PyObject *o, int32_t dim, float &scale) {
    if (o == Py_None) scale = static_cast<float>(1.0 / std::sqrt(static_cast<double>(dim)));
    else if (PyFloat_CheckExact(o)) scale = static_cast<float>(PyFloat_AS_DOUBLE(o));
    else return false;
    return true;
}

// mask or None, for n tokens
bool mask_of(PyObject *o, const Held &ix, int64_t n, const uint32_t *&mask, int32_t &words) {
    mask = nullptr;
    words = 0;
    if (o == Py_None) return true;
    mask = reinterpret_cast<const uint32_t *>(ints(o, 0, ix.gpu));
    if (!mask) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.dim() != 2 || t.size(0) != n || t.size(1) > INT32_MAX) return false;
    words = static_cast<int32_t>(t.size(1));
    return true;
}

// (.., mask or None, scale or None, n_sink, window)
PyObject *window_attention(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    QueryArgs a;
    float scale;
    int64_t sink, window;
    const uint32_t *mask;
    int32_t words;
    if (!p_window_attention_workspace_bytes || !p_window_attention || n_args != 12 || !queries(args, a) || !scale_of(args[9], pool_of(a.pool)->dim, scale) || !integer(args[10], 0, INT32_MAX, sink) || !integer(args[11], 1, INT32_MAX, window) ||
        !mask_of(args[8], a.ix, a.q->size(0), mask, words))
        Py_RETURN_NONE;
    const int64_t n = a.q->size(0), heads = a.q->size(1);
    const int32_t max_q = static_cast<int32_t>(a.max_q), H = static_cast<int32_t>(heads), n_sink = static_cast<int32_t>(sink), w = static_cast<int32_t>(window);
    const auto *pool = pool_of(a.pool);
    const auto *ix = index_of(a.ix);
    at::Tensor out = at::empty({n, heads, pool->dim}, a.q->options()), lse = at::empty({n, heads}, a.q->options().dtype(at::kFloat)), ws;
    const size_t need = p_window_attention_workspace_bytes(pool, ix, n, max_q, H, n_sink, w, mask != nullptr, a.max_len);
    if (need) ws = bytes_like(*a.q, need);
    const tbn_status st = unlocked([&] {
        return p_window_attention(a.q->data_ptr(), a.stride, out.data_ptr(), floats(lse), pool, ix, a.cu, n, max_q, H, n_sink, w, mask, words, a.max_len, scale,
                                  need ? ws.data_ptr() : nullptr, need, stream());
    });
    return result(st, two, out, lse);
    END_HANDLE_TH_ERRORS
}

PyObject *kv4_attention(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    QueryArgs a;
    float scale;
    int64_t sink, window;
    const uint32_t *mask;
    int32_t words;
    if (!p_kv4_attention_workspace_bytes || !p_kv4_attention || n_args != 12 || !queries(args, a, true) || !scale_of(args[9], pool4_of(a.pool)->dim, scale) || !integer(args[10], 0, INT32_MAX, sink) ||
        !integer(args[11], 0, INT32_MAX, window) || !mask_of(args[8], a.ix, a.q->size(0), mask, words))
        Py_RETURN_NONE;
    const int64_t n = a.q->size(0), heads = a.q->size(1);
    const int32_t max_q = static_cast<int32_t>(a.max_q), H = static_cast<int32_t>(heads), n_sink = static_cast<int32_t>(sink), w = static_cast<int32_t>(window);
    const auto *pool = pool4_of(a.pool);
    const auto *ix = index_of(a.ix);
    at::Tensor out = at::empty({n, heads, pool->dim}, a.q->options()), lse = at::empty({n, heads}, a.q->options().dtype(at::kFloat)), ws;
    const size_t need = p_kv4_attention_workspace_bytes(pool, ix, a.dt, n, max_q, H, n_sink, w, mask != nullptr, a.max_len);
    if (need) ws = bytes_like(*a.q, need);
    const tbn_status st = unlocked([&] {
        return p_kv4_attention(a.q->data_ptr(), a.stride, a.dt, out.data_ptr(), floats(lse), pool, ix, a.cu, n, max_q, H, n_sink, w, mask, words, a.max_len, scale,
                               need ? ws.data_ptr() : nullptr, need, stream());
    });
    return result(st, two, out, lse);
    END_HANDLE_TH_ERRORS
}

// (.., mask or None, scale or None)
PyObject *tree_attention(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    QueryArgs a;
    float scale;
    const uint32_t *mask;
    int32_t words;
    if (n_args != 10 || !queries(args, a) || !scale_of(args[9], pool_of(a.pool)->dim, scale) || !mask_of(args[8], a.ix, a.q->size(0), mask, words)) Py_RETURN_NONE;
    const int64_t n = a.q->size(0), heads = a.q->size(1);
    const auto *pool = pool_of(a.pool);
    const auto *ix = index_of(a.ix);
    at::Tensor out = at::empty({n, heads, pool->dim}, a.q->options()), lse = at::empty({n, heads}, a.q->options().dtype(at::kFloat)), ws;
    const size_t need = p_tree_attention_workspace_bytes(pool, ix, n, static_cast<int32_t>(a.max_q), static_cast<int32_t>(heads), a.max_len);
    if (need) ws = bytes_like(*a.q, need);
    const tbn_status st = unlocked([&] {
        return p_tree_attention(a.q->data_ptr(), a.stride, out.data_ptr(), floats(lse), pool, ix, a.cu, n, static_cast<int32_t>(a.max_q),
                                static_cast<int32_t>(heads), mask, words, a.max_len, scale,
                                need ? ws.data_ptr() : nullptr, need, stream());
    });
    return result(st, two, out, lse);
    END_HANDLE_TH_ERRORS
}

// (.., n_select, n_sink, n_recent)
PyObject *block_select(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    QueryArgs a;
    int64_t select, sink, recent;
    if (n_args != 11 || !queries(args, a) || !integer(args[8], 1, 4096, select) || !integer(args[9], 0, 4096, sink) || !integer(args[10], 1, 4096, recent)) Py_RETURN_NONE;
    const int64_t n = a.q->size(0), heads = a.q->size(1);
    const auto *pool = pool_of(a.pool);
    const auto *ix = index_of(a.ix);
    at::Tensor picks = at::empty({n, pool->kv_heads, select}, a.q->options().dtype(at::kInt)), ws;
    const size_t need = p_block_select_workspace_bytes(pool, ix, n, static_cast<int32_t>(a.max_q), static_cast<int32_t>(heads), a.max_len);
    if (need) ws = bytes_like(*a.q, need);
    const tbn_status st = unlocked([&] {
        return p_block_select(a.q->data_ptr(), a.stride, static_cast<int32_t *>(picks.data_ptr()), pool, ix, a.cu, n, static_cast<int32_t>(a.max_q),
                              static_cast<int32_t>(heads), static_cast<int32_t>(select), static_cast<int32_t>(sink), static_cast<int32_t>(recent), a.max_len,
                              need ? ws.data_ptr() : nullptr, need, stream());
    });
    return result(st, one, picks, picks);
    END_HANDLE_TH_ERRORS
}

// (.., picks, scale or None); max_len is not looked at
PyObject *block_attention(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    QueryArgs a;
    float scale;
    if (n_args != 10 || !queries(args, a) || !scale_of(args[9], pool_of(a.pool)->dim, scale)) Py_RETURN_NONE;
    const int64_t n = a.q->size(0), heads = a.q->size(1);
    const auto *pool = pool_of(a.pool);
    const auto *ix = index_of(a.ix);
    const int32_t *picks = ints(args[8], 0, a.ix.gpu);
    if (!picks) Py_RETURN_NONE;
    const at::Tensor &t = THPVariable_Unpack(args[8]);
    if (t.dim() != 3 || t.size(0) != n || t.size(1) != pool->kv_heads || t.size(2) < 1 || t.size(2) > 4096) Py_RETURN_NONE;
    const int32_t select = static_cast<int32_t>(t.size(2));
    at::Tensor out = at::empty({n, heads, pool->dim}, a.q->options()), lse = at::empty({n, heads}, a.q->options().dtype(at::kFloat)), ws;
    const size_t need = p_block_attention_workspace_bytes(pool, ix, n, static_cast<int32_t>(a.max_q), static_cast<int32_t>(heads), select);
    if (need) ws = bytes_like(*a.q, need);
    const tbn_status st = unlocked([&] {
        return p_block_attention(a.q->data_ptr(), a.stride, out.data_ptr(), floats(lse), pool, ix, a.cu, n, static_cast<int32_t>(a.max_q),
                                 static_cast<int32_t>(heads), picks, select, scale, need ? ws.data_ptr() : nullptr, need, stream());
    });
    return result(st, two, out, lse);
    END_HANDLE_TH_ERRORS
}

// float32 (tokens, vocab) with dense rows
const at::Tensor *probabilities(PyObject *o, int64_t &stride) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    constexpr c10::DispatchKeySet kWrapped({c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::FuncTorchGradWrapper,
                                            c10::DispatchKey::Functionalize, c10::DispatchKey::Python});
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || t.dim() != 2 || t.scalar_type() != at::kFloat || t.key_set().has_any(kWrapped)) return nullptr;
    const int64_t n = t.size(0), v = t.size(1);
    if (n < 1 || v < 1 || t.stride(1) != 1 || (n > 1 && t.stride(0) < v)) return nullptr;
    stride = n > 1 ? t.stride(0) : v;
    return &t;
}

// (target, tokens, u, cu_q, max_q, draft or None, parents or None)
PyObject *verify(PyObject *, PyObject *const *args, Py_ssize_t n_args) {
    HANDLE_TH_ERRORS
    int64_t ps, qs = 0, most;
    if (!p_verify_workspace_bytes || !p_verify || n_args != 7 || !ordinary_context()) Py_RETURN_NONE;
    const at::Tensor *p = probabilities(args[0], ps), *q = nullptr;
    if (!p || !integer(args[4], 0, 2048, most)) Py_RETURN_NONE;   // more tokens, or sequences, get no memory: the wrapper raises the library's error
    const int64_t n = p->size(0), vocab = p->size(1), gpu = p->device().index();
    const int32_t *tokens = ints(args[1], n, gpu), *cu = ints(args[3], 2, gpu), *parents = nullptr;
    const at::Tensor *u = plain(args[2], at::kFloat, *p);
    if (!tokens || !cu || !u || u->numel() < n) Py_RETURN_NONE;
    if (args[5] != Py_None && (!(q = probabilities(args[5], qs)) || q->sizes() != p->sizes() || q->device() != p->device())) Py_RETURN_NONE;
    if (args[6] != Py_None && !(parents = ints(args[6], n, gpu))) Py_RETURN_NONE;
    const int64_t n_seqs = THPVariable_Unpack(args[3]).numel() - 1;
    if (n_seqs > 8192) Py_RETURN_NONE;
    const auto options = THPVariable_Unpack(args[3]).options();
    at::Tensor picks = at::empty({n_seqs, most}, options), counts = at::empty({n_seqs}, options), next = at::empty({n_seqs}, options), ws;
    const int32_t max_q = static_cast<int32_t>(most), seqs = static_cast<int32_t>(n_seqs);
    const size_t need = p_verify_workspace_bytes(n, max_q, seqs, vocab);
    if (need) ws = bytes_like(*p, need);
    const tbn_status st = unlocked([&] {
        return p_verify(floats(*p), ps, q ? floats(*q) : nullptr, qs, tokens, parents, floats(*u), cu, n, max_q, seqs, vocab, static_cast<int32_t *>(picks.data_ptr()),
                        static_cast<int32_t *>(counts.data_ptr()), static_cast<int32_t *>(next.data_ptr()), need ? ws.data_ptr() : nullptr, need, stream());
    });
    if (st != TBN_OK) return result(st, one, picks, picks);
    PyObject *a = THPVariable_Wrap(picks), *b = THPVariable_Wrap(counts), *c = THPVariable_Wrap(next);
    PyObject *r = a && b && c ? PyTuple_Pack(3, a, b, c) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    Py_XDECREF(c);
    return r;
    END_HANDLE_TH_ERRORS
}

// (raise, {name: address})
PyObject *init(PyObject *, PyObject *args) {
    PyObject *raise, *table;
    if (!PyArg_ParseTuple(args, "OO!", &raise, &PyDict_Type, &table)) return nullptr;
    bool ok = true;
    auto take = [&](auto &fn, const char *name) {
        PyObject *a = PyDict_GetItemString(table, name);
        void *p = a && PyLong_Check(a) ? PyLong_AsVoidPtr(a) : nullptr;
        ok = ok && p;
        fn = reinterpret_cast<std::decay_t<decltype(fn)>>(p);
    };
    take(p_pack_workspace_bytes, "tbn_pack_workspace_bytes");
    take(p_pack_tile, "tbn_pack_tile");
    take(p_linear_forward, "tbn_linear_forward");
    take(p_conv2d_forward, "tbn_conv2d_forward");
    take(p_coltiled_workspace_bytes, "tbn_linear_coltiled_workspace_bytes");
    take(p_coltiled_forward, "tbn_linear_coltiled_forward");
    take(p_sign_pack, "tbn_sign_pack");
    take(p_forward_binact, "tbn_linear_forward_binact");
    take(p_kv_workspace_bytes, "tbn_kv_workspace_bytes");
    take(p_kv_reserve, "tbn_kv_reserve");
    take(p_kv_fork, "tbn_kv_fork");
    take(p_kv_release, "tbn_kv_release");
    take(p_kv_copy_pages, "tbn_kv_copy_pages");
    take(p_kv_append, "tbn_kv_append");
    take(p_kv_keep, "tbn_kv_keep");
    take(p_tree_attention_workspace_bytes, "tbn_tree_attention_workspace_bytes");
    take(p_tree_attention, "tbn_tree_attention");
    take(p_block_select_workspace_bytes, "tbn_block_select_workspace_bytes");
    take(p_block_select, "tbn_block_select");
    take(p_block_attention_workspace_bytes, "tbn_block_attention_workspace_bytes");
    take(p_block_attention, "tbn_block_attention");
    // A table may leave these out: they stay as they were, and without an address their calls are not taken.
    auto take_if = [&](auto &fn, const char *name) {
        if (PyDict_GetItemString(table, name)) take(fn, name);
    };
    take_if(p_window_attention_workspace_bytes, "tbn_window_attention_workspace_bytes");
    take_if(p_window_attention, "tbn_window_attention");
    take_if(p_kv4_append, "tbn_kv4_append");
    take_if(p_kv4_read, "tbn_kv4_read");
    take_if(p_kv4_copy_pages, "tbn_kv4_copy_pages");
    take_if(p_kv4_keep, "tbn_kv4_keep");
    take_if(p_kv4_attention_workspace_bytes, "tbn_kv4_attention_workspace_bytes");
    take_if(p_kv4_attention, "tbn_kv4_attention");
    take_if(p_verify_workspace_bytes, "tbn_verify_workspace_bytes");
    take_if(p_verify, "tbn_verify");
    if (!ok) {
        PyErr_SetString(PyExc_ImportError, "_tbn_host: an entry point of the library is missing");
        return nullptr;
    }
    Py_INCREF(raise);
    Py_XDECREF(g_raise);
    g_raise = raise;
    Py_RETURN_NONE;
}

#define TBN_FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {TBN_FAST(linear_forward), TBN_FAST(conv2d_forward), TBN_FAST(linear_coltiled_forward), TBN_FAST(sign_pack),
                         TBN_FAST(linear_forward_binact), TBN_FAST(pack_tile),
                         TBN_FAST(kv_reserve), TBN_FAST(kv_fork), TBN_FAST(kv_release), TBN_FAST(kv_copy_pages), TBN_FAST(kv_append), TBN_FAST(kv_keep),
                         TBN_FAST(tree_attention), TBN_FAST(window_attention), TBN_FAST(kv4_append), TBN_FAST(kv4_read),
                         TBN_FAST(kv4_copy_pages), TBN_FAST(kv4_keep), TBN_FAST(kv4_attention), TBN_FAST(verify),
                         TBN_FAST(block_select), TBN_FAST(block_attention), {"init", init, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tbn_host", "plain calls of the binding on C++ tensors", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tbn_host(void) { return PyModule_Create(&module); }
