// The calls of the Python binding that a decode step or a small product makes, without an interpreter between the tensors and the C ABI.
//
// A single product from Python was bound by its marshalling: attribute look-ups on tensors, checks and the conversion of thirteen
// arguments took 2 to 3 us of a call whose kernel takes 2 to 5.  Here an argument is looked at where it lies, in the tensor's own structure: W1A2 16 x 256 x 512
// (pack + product) 10.9 -> 8.2 us, W2A2 1 x 11008 x 4096 from codes 6.2 -> 4.6, of which the kernel takes 4.4.  Outputs that are not given are allocated here:
// handed over, such a call took 0.1 to 0.3 us longer than without this module (W2A2 1 x 1024 x 1024 6.9 -> 7.1 us, from codes 7.3 -> 7.6, quantisation 6.7 -> 7.0), now 5.0, 5.0 and 4.5.
//
// Every function takes the arguments of the Python function of the same name in binding.py and has that function as its `general` form: whatever
// is not the plain case (anything that is not a torch.Tensor, an integer of another type, an output that cannot be allocated, a check
// that fails, an unknown keyword, a torch-function mode, a process forked from one that uses the GPU, the library not loaded yet) is handed to it with the very arguments, so that
// results and errors are its own.  A status other than 0 goes to binding.py's _check, on the same thread.  As through ctypes, the interpreter's lock is
// released around the call.
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/device_lazy_init.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>

#include <cmath>
#include <cstring>

#include "../../include/apmm.h"
#include "apmm_call_guard.h"

namespace {

struct Library {
    decltype(&apmm_packed_bytes) packed_bytes;
    decltype(&apmm_packed_activation_bytes) packed_activation_bytes;
    decltype(&apmm_pack_weights) pack_weights;
    decltype(&apmm_pack_activations) pack_activations;
    decltype(&apmm_quantize_pack_activations) quantize_pack_activations;
    decltype(&apmm_gemm_ex) gemm_ex;
    decltype(&apmm_gemm_from_codes) gemm_from_codes;
    decltype(&apmm_kv_write) kv_write;
    decltype(&apmm_kv_read) kv_read;
    decltype(&apmm_kv_attention) kv_attention;
    decltype(&apmm_kv_attention_workspace_bytes) kv_attention_workspace_bytes;
    decltype(&apmm_rotary) rotary;
    decltype(&apmm_kv_write_rotary) kv_write_rotary;
    decltype(&apmm_kv_weights) kv_weights;
    decltype(&apmm_kv_weights_workspace_bytes) kv_weights_workspace_bytes;
    decltype(&apmm_kv_evict) kv_evict;
    decltype(&apmm_kv_evict_workspace_bytes) kv_evict_workspace_bytes;
    decltype(&apmm_w4_packed_bytes) w4_packed_bytes;
    decltype(&apmm_w4_workspace_bytes) w4_workspace_bytes;
    decltype(&apmm_w4_gemm) w4_gemm;
};
constexpr int kLibraryFunctions = 20;
Library lib = {};
bool loaded = false;
PyObject *check = nullptr;  // binding.py's _check

constexpr int kMaxArgs = 15;
enum Function { kPackWeights, kPackActivations, kQuantize, kGemm, kFromCodes, kKvWrite, kKvRead, kKvAttention, kRotary, kKvWriteRotary, kKvWeights, kKvEvict, kW4Gemm, kFunctions };
struct Signature {
    const char *name;
    int count, required;
    const char *args[kMaxArgs];
    PyObject *keys[kMaxArgs];  // the interned names
    PyObject *general;
};
Signature signatures[kFunctions] = {
    {"apmm_pack_weights", 3, 2, {"w_codes", "q", "out"}, {}, nullptr},
    {"apmm_pack_activations", 3, 2, {"a_codes", "p", "out"}, {}, nullptr},
    {"apmm_quantize_pack_activations", 4, 2, {"x_f16", "p", "out", "scale_out"}, {}, nullptr},
    {"apmm_gemm", 15, 7,
     {"M", "N", "K", "p", "q", "a_packed", "w_packed", "want_i32", "want_f16", "w_scale", "a_scale", "c_i32", "c_f16", "workspace", "algo"}, {}, nullptr},
    {"apmm_gemm_from_codes", 12, 5, {"a_codes", "N", "p", "q", "w_packed", "want_i32", "want_f16", "w_scale", "a_scale", "c_i32", "c_f16", "workspace"}, {}, nullptr},
    {"apmm_kv_write", 7, 6, {"k", "v", "codes", "scales", "page_table", "lengths", "starts"}, {}, nullptr},
    {"apmm_kv_read", 8, 5, {"codes", "scales", "page_table", "lengths", "tokens", "starts", "k_out", "v_out"}, {}, nullptr},
    {"apmm_kv_attention", 11, 5, {"q", "codes", "scales", "page_table", "lengths", "starts", "window", "sinks", "scale", "out", "workspace"}, {}, nullptr},
    {"apmm_rotary", 7, 3, {"x", "positions", "frequencies", "interleaved", "magnitude", "inverse", "out"}, {}, nullptr},
    {"apmm_kv_write_rotary", 13, 8,
     {"q", "k", "v", "codes", "scales", "page_table", "lengths", "frequencies", "starts", "positions", "interleaved", "magnitude", "q_out"}, {}, nullptr},
    {"apmm_kv_weights", 12, 6, {"q", "codes", "scales", "page_table", "lengths", "weights", "starts", "window", "sinks", "scale", "decay", "workspace"}, {}, nullptr},
    {"apmm_kv_evict", 13, 7,
     {"codes", "scales", "page_table", "lengths", "weights", "budget", "to_table", "sinks", "recent", "kept", "to_weights", "to_lengths", "workspace"}, {}, nullptr},
    {"apmm_w4_gemm", 6, 4, {"x", "packed", "N", "group", "out", "workspace"}, {}, nullptr},
};

// Arguments by place, null where not given; false: not the plain case.
bool place(const Signature &s, PyObject *const *args, Py_ssize_t nargs, PyObject *names, PyObject **out)
{
    if (!loaded || nargs > s.count || at::impl::torch_function_mode_enabled() || torch::utils::is_device_in_bad_fork(at::kCUDA)) return false;
    for (int i = 0; i < s.count; ++i) out[i] = i < nargs ? args[i] : nullptr;
    const Py_ssize_t named = names ? PyTuple_GET_SIZE(names) : 0;
    for (Py_ssize_t i = 0; i < named; ++i) {
        PyObject *key = PyTuple_GET_ITEM(names, i);
        int at = (int)nargs;
        while (at < s.count && s.keys[at] != key) ++at;
        if (at == s.count || out[at]) return false;
        out[at] = args[nargs + i];
    }
    for (int i = 0; i < s.required; ++i)
        if (!out[i]) return false;
    return true;
}

bool integer(PyObject *o, int64_t lo, int64_t hi, int64_t &v)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return !overflow && v >= lo && v <= hi;
}
constexpr int64_t kAny = INT64_MAX;

bool flag(PyObject *o, bool absent, bool &v)
{
    v = o ? o == Py_True : absent;
    return !o || o == Py_True || o == Py_False;
}

bool given(PyObject *o) { return o && o != Py_None; }
const at::Tensor *tensor(PyObject *o)
{
    if (!given(o) || !THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.defined() && t.is_cuda() && t.layout() == at::kStrided && t.has_storage() ? &t : nullptr;
}
// null pointer for an absent tensor; false: not the plain case
bool address(PyObject *o, void *&p)
{
    p = nullptr;
    if (!given(o)) return true;
    const at::Tensor *t = tensor(o);
    if (t) p = t->data_ptr();
    return t != nullptr;
}
bool matrix(const at::Tensor *t, at::ScalarType type) { return t && t->scalar_type() == type && t->dim() == 2 && t->is_contiguous(); }
bool scale_ok(PyObject *o, int64_t n)
{
    if (!given(o)) return true;
    const at::Tensor *t = tensor(o);
    return t && t->scalar_type() == at::kHalf && t->numel() == n && t->is_contiguous();
}
size_t bytes(const at::Tensor &t) { return t.nbytes(); }
void *stream() { return c10::hip::getCurrentHIPStream().stream(); }

PyObject *general(const Signature &s, PyObject *const *args, Py_ssize_t nargs, PyObject *names)
{
    if (!s.general) {
        PyErr_SetString(PyExc_RuntimeError, "apmm: the general function is not set");
        return nullptr;
    }
    return PyObject_Vectorcall(s.general, args, (size_t)nargs, names);
}

template <class Call>
bool called(Call call) { return call_and_check(check, call); }

// An output by the place of its argument: the caller's, or a new tensor as the Python function allocates it.  Nothing is given back by a destructor:
// a thread that ends inside the call is unwound without the interpreter's lock.
struct Output {
    PyObject *object = nullptr;  // None where neither given nor wanted
    void *address = nullptr;
    bool made = false;
};
// false: not the plain case
bool output(Output &o, PyObject *arg, bool wanted, const at::Tensor &like, at::IntArrayRef size, at::ScalarType type)
{
    o.object = arg ? arg : Py_None;
    if (given(arg) || !wanted) return address(arg, o.address);
    at::Tensor t;
    bool allocated;
    Py_BEGIN_ALLOW_THREADS
    allocated = end_exceptions([&] { t = at::empty(size, like.options().dtype(type)); return true; }, [] { return false; });
    Py_END_ALLOW_THREADS
    if (!allocated) return false;
    o.object = THPVariable_Wrap(std::move(t));
    o.made = o.object != nullptr;
    if (!o.made) {
        PyErr_Clear();
        return false;
    }
    return address(o.object, o.address);
}
// The result of a call that went well (one output, or two as a tuple), or what stands for one that did not: 1 and the result, else `done`
int result_of(int done, Output &a, Output *b, PyObject *&result)
{
    if (done == 1) {
        result = b ? PyTuple_Pack(2, a.object, b->object) : a.object;
        if (!b) Py_INCREF(result);
        if (!result) done = -1;
    }
    if (a.made) Py_DECREF(a.object);
    if (b && b->made) Py_DECREF(b->object);
    return done;
}
int64_t at_least_one(size_t n) { return n > 1 ? (int64_t)n : 1; }

// Each returns 1 and the result, 0 for the general form, -1 with an error set.
int pack(Function f, PyObject **v, PyObject *&result)
{
    int64_t bits;
    const at::Tensor *codes = tensor(v[0]);
    if (!matrix(codes, at::kByte) || !integer(v[1], 1, 8, bits) || (given(v[2]) && !tensor(v[2]))) return 0;
    const int64_t rows = codes->size(0), K = codes->size(1);
    const bool weights = f == kPackWeights;
    const size_t need = (weights ? lib.packed_bytes : lib.packed_activation_bytes)(rows, K, (int)bits);
    if (given(v[2]) && bytes(*tensor(v[2])) < need) return 0;
    const uint8_t *src = static_cast<const uint8_t *>(codes->data_ptr());
    Output out;
    if (!output(out, v[2], true, *codes, {at_least_one(need)}, at::kByte)) return result_of(0, out, nullptr, result);
    void *s = stream();
    const bool went = called([&] { return (weights ? lib.pack_weights : lib.pack_activations)(src, rows, K, (int)bits, out.address, s); });
    return result_of(went ? 1 : -1, out, nullptr, result);
}

int quantize(PyObject **v, PyObject *&result)
{
    int64_t p;
    const at::Tensor *x = tensor(v[0]);
    if (!matrix(x, at::kHalf) || !integer(v[1], 1, 8, p) || (given(v[2]) && !tensor(v[2])) || (given(v[3]) && !tensor(v[3]))) return 0;
    const int64_t M = x->size(0), K = x->size(1);
    const size_t need = lib.packed_activation_bytes(M, K, (int)p);
    if (given(v[2]) && bytes(*tensor(v[2])) < need) return 0;
    if (given(v[3]) && (tensor(v[3])->scalar_type() != at::kHalf || tensor(v[3])->numel() < M)) return 0;
    const uint16_t *src = static_cast<const uint16_t *>(x->data_ptr());
    Output out, scale;
    if (!output(out, v[2], true, *x, {at_least_one(need)}, at::kByte) || !output(scale, v[3], true, *x, {M}, at::kHalf)) return result_of(0, out, &scale, result);
    void *s = stream();
    const bool went = called([&] { return lib.quantize_pack_activations(src, M, K, (int)p, out.address, static_cast<uint16_t *>(scale.address), s); });
    return result_of(went ? 1 : -1, out, &scale, result);
}

int gemm(PyObject **v, PyObject *&result)
{
    int64_t M, N, K, p, q, algo = APMM_ALGO_AUTO;
    bool want_i32, want_f16;
    void *a, *w, *ws, *as, *space;
    if (!integer(v[0], 0, kAny, M) || !integer(v[1], 0, kAny, N) || !integer(v[2], 0, kAny, K) || !integer(v[3], 0, 255, p) || !integer(v[4], 0, 255, q) ||
        !flag(v[7], true, want_i32) || !flag(v[8], false, want_f16) || !given(v[5]) || !given(v[6]) || (v[14] && !integer(v[14], 0, 255, algo)) ||
        !scale_ok(v[9], N) || !scale_ok(v[10], M) || !address(v[5], a) || !address(v[6], w) || !address(v[9], ws) || !address(v[10], as) || !address(v[13], space))
        return 0;
    const size_t room = given(v[13]) ? bytes(*tensor(v[13])) : 0;
    const at::Tensor &like = *tensor(v[5]);
    Output ci, cf;
    if (!output(ci, v[11], want_i32, like, {M, N}, at::kInt) || !output(cf, v[12], want_f16, like, {M, N}, at::kHalf)) return result_of(0, ci, &cf, result);
    void *s = stream();
    const bool went = called([&] {
        return lib.gemm_ex(M, N, K, (int)p, (int)q, a, w, static_cast<int32_t *>(ci.address), static_cast<uint16_t *>(cf.address), static_cast<const uint16_t *>(ws),
                           static_cast<const uint16_t *>(as), space, room, s, (int)algo);
    });
    return result_of(went ? 1 : -1, ci, &cf, result);
}

int from_codes(PyObject **v, PyObject *&result)
{
    int64_t N, p, q;
    bool want_i32, want_f16;
    void *w, *ws, *as, *space;
    const at::Tensor *codes = tensor(v[0]);
    if (!matrix(codes, at::kByte) || !integer(v[1], 0, kAny, N) || !integer(v[2], 0, 255, p) || !integer(v[3], 0, 255, q) || !given(v[4]) ||
        !flag(v[5], true, want_i32) || !flag(v[6], false, want_f16) || !address(v[4], w) || !address(v[7], ws) || !address(v[8], as) || !address(v[11], space))
        return 0;
    const int64_t M = codes->size(0), K = codes->size(1);
    const uint8_t *a = static_cast<const uint8_t *>(codes->data_ptr());
    const size_t room = given(v[11]) ? bytes(*tensor(v[11])) : 0;
    Output ci, cf;
    if (!output(ci, v[9], want_i32, *codes, {M, N}, at::kInt) || !output(cf, v[10], want_f16, *codes, {M, N}, at::kHalf)) return result_of(0, ci, &cf, result);
    void *s = stream();
    const bool went = called([&] {
        return lib.gemm_from_codes(M, N, K, (int)p, (int)q, a, w, static_cast<int32_t *>(ci.address), static_cast<uint16_t *>(cf.address), static_cast<const uint16_t *>(ws),
                                   static_cast<const uint16_t *>(as), space, room, s);
    });
    return result_of(went ? 1 : -1, ci, &cf, result);
}

// The four-bit cache: its two tensors, the batch and rows of a call as binding.py checks them
bool kv_cache(PyObject *codes_arg, PyObject *scales_arg, apmm_kv_cache &c)
{
    const at::Tensor *codes = tensor(codes_arg), *scales = tensor(scales_arg);
    if (!codes || !scales || codes->scalar_type() != at::kByte || (scales->scalar_type() != at::kHalf && scales->scalar_type() != at::kBFloat16) || codes->dim() != 4 ||
        scales->dim() != 4 || !codes->is_contiguous() || !scales->is_contiguous() || codes->get_device() != scales->get_device() ||
        codes->get_device() != c10::hip::getCurrentHIPStream().device_index())
        return false;
    const int64_t pages = codes->size(0), heads = codes->size(1), page_size = scales->size(3);
    if (scales->size(0) != pages || scales->size(1) != heads || codes->size(2) != 2 || scales->size(2) != 2 || page_size < 1 || codes->size(3) < 1 || codes->size(3) * 2 % page_size) return false;
    const int64_t head_dim = codes->size(3) * 2 / page_size;
    if (heads > INT32_MAX || page_size > INT32_MAX || head_dim > INT32_MAX) return false;
    c = {codes->data_ptr(), scales->data_ptr(), pages, (int)page_size, (int)heads, (int)head_dim, scales->scalar_type() == at::kHalf ? APMM_F16 : APMM_BF16};
    return true;
}
bool kv_indices(const at::Tensor *t, int64_t dim, int device)
{
    return t && t->scalar_type() == at::kInt && t->dim() == dim && t->get_device() == device && (t->size(dim - 1) <= 1 || t->stride(dim - 1) == 1);
}
bool kv_batch(PyObject *codes, PyObject *table_arg, PyObject *lengths_arg, PyObject *starts_arg, int64_t tokens, apmm_kv_batch &b)
{
    const int device = tensor(codes)->get_device();
    const at::Tensor *table = tensor(table_arg), *lengths = tensor(lengths_arg), *starts = tensor(starts_arg);
    if (!kv_indices(table, 2, device) || !kv_indices(lengths, 1, device) || (given(starts_arg) && !kv_indices(starts, 1, device))) return false;
    const int64_t n = lengths->size(0);
    if (n > INT32_MAX || table->size(0) != n || (starts ? starts->size(0) != n + 1 : tokens != n)) return false;
    b = {(int)n, tokens, static_cast<const int32_t *>(lengths->data_ptr()), starts ? static_cast<const int32_t *>(starts->data_ptr()) : nullptr,
         static_cast<const int32_t *>(table->data_ptr()), n > 1 ? table->stride(0) : table->size(1), table->size(1)};
    return true;
}
bool kv_rows(const at::Tensor *t, PyObject *scales_arg, int64_t heads, int64_t head_dim, int64_t tokens)
{
    const at::Tensor *scales = tensor(scales_arg);
    return t && t->scalar_type() == scales->scalar_type() && t->get_device() == scales->get_device() && t->dim() == 3 && t->size(0) == tokens && t->size(1) == heads &&
           t->size(2) == head_dim && t->stride(2) == 1;
}

int kv_write(PyObject **v, PyObject *&result)
{
    apmm_kv_cache c;
    apmm_kv_batch b;
    const at::Tensor *k = tensor(v[0]), *x = tensor(v[1]);
    if (!k || !x || k->dim() != 3 || !kv_cache(v[2], v[3], c) || !kv_batch(v[2], v[4], v[5], v[6], k->size(0), b) || !kv_rows(k, v[3], c.kv_heads, c.head_dim, b.tokens) ||
        !kv_rows(x, v[3], c.kv_heads, c.head_dim, b.tokens))
        return 0;
    void *s = stream();
    if (!called([&] { return lib.kv_write(&c, &b, k->data_ptr(), k->stride(0), k->stride(1), x->data_ptr(), x->stride(0), x->stride(1), s); })) return -1;
    Py_INCREF(Py_None);
    result = Py_None;
    return 1;
}

int kv_read(PyObject **v, PyObject *&result)
{
    apmm_kv_cache c;
    apmm_kv_batch b;
    int64_t tokens;
    if (!kv_cache(v[0], v[1], c) || !integer(v[4], 0, INT32_MAX, tokens) || !kv_batch(v[0], v[2], v[3], v[5], tokens, b)) return 0;
    for (int i = 6; i < 8; ++i)
        if (given(v[i]) && !kv_rows(tensor(v[i]), v[1], c.kv_heads, c.head_dim, tokens)) return 0;
    const at::Tensor &like = *tensor(v[1]);
    Output k, x;
    if (!output(k, v[6], true, like, {tokens, c.kv_heads, c.head_dim}, like.scalar_type()) || !output(x, v[7], true, like, {tokens, c.kv_heads, c.head_dim}, like.scalar_type()))
        return result_of(0, k, &x, result);
    const at::Tensor &tk = *tensor(k.object), &tx = *tensor(x.object);
    void *s = stream();
    const bool went = called([&] { return lib.kv_read(&c, &b, k.address, tk.stride(0), tk.stride(1), x.address, tx.stride(0), tx.stride(1), s); });
    return result_of(went ? 1 : -1, k, &x, result);
}

int kv_attention(PyObject **v, PyObject *&result)
{
    apmm_kv_cache c;
    apmm_kv_batch b;
    int64_t window = 0, sinks = 0;
    const at::Tensor *q = tensor(v[0]);
    if (!q || q->dim() != 3 || !kv_cache(v[1], v[2], c) || !kv_batch(v[1], v[3], v[4], v[5], q->size(0), b) || q->size(1) > INT32_MAX ||
        !kv_rows(q, v[2], q->size(1), c.head_dim, b.tokens) || (given(v[9]) && !kv_rows(tensor(v[9]), v[2], q->size(1), c.head_dim, b.tokens)) ||
        (v[6] && !integer(v[6], -kAny, kAny, window)) || (v[7] && !integer(v[7], -kAny, kAny, sinks)) || (given(v[8]) && !PyFloat_CheckExact(v[8])) ||
        (given(v[10]) && (!tensor(v[10]) || !tensor(v[10])->is_contiguous() || tensor(v[10])->get_device() != q->get_device())))
        return 0;
    const int heads = (int)q->size(1);
    const float scale = (float)(given(v[8]) ? PyFloat_AS_DOUBLE(v[8]) : 1.0 / std::sqrt((double)c.head_dim));
    const size_t need = given(v[10]) ? 0 : lib.kv_attention_workspace_bytes(&c, &b, heads);
    Output out, work;
    int done = output(out, v[9], true, *q, {b.tokens, heads, c.head_dim}, q->scalar_type()) && output(work, v[10], need != 0, *q, {(int64_t)need}, at::kByte);
    if (done) {
        const at::Tensor &to = *tensor(out.object);
        const size_t room = work.address ? bytes(*tensor(work.object)) : 0;
        void *s = stream();
        const bool went = called([&] {
            return lib.kv_attention(&c, &b, heads, q->data_ptr(), q->stride(0), q->stride(1), out.address, to.stride(0), to.stride(1), scale, window, sinks, work.address, room, s);
        });
        done = went ? 1 : -1;
    }
    if (work.made) Py_DECREF(work.object);
    return result_of(done, out, nullptr, result);
}

bool half_type(const at::Tensor *t) { return t && (t->scalar_type() == at::kHalf || t->scalar_type() == at::kBFloat16); }
int dtype_of(const at::Tensor &t) { return t.scalar_type() == at::kHalf ? APMM_F16 : APMM_BF16; }
bool number(PyObject *o, double absent, float &v)
{
    if (o && !PyFloat_CheckExact(o)) return false;
    v = (float)(o ? PyFloat_AS_DOUBLE(o) : absent);
    return true;
}
bool dense_last(const at::Tensor &t) { return t.size(t.dim() - 1) <= 1 || t.stride(t.dim() - 1) == 1; }
bool rotation(PyObject *frequencies_arg, PyObject *interleaved_arg, PyObject *magnitude_arg, int device, apmm_rotation &r)
{
    const at::Tensor *f = tensor(frequencies_arg);
    bool interleaved;
    if (!f || f->scalar_type() != at::kDouble || f->dim() != 1 || !f->is_contiguous() || f->get_device() != device || !flag(interleaved_arg, false, interleaved) ||
        !number(magnitude_arg, 1.0, r.magnitude))
        return false;
    r.frequencies = static_cast<const double *>(f->data_ptr());
    r.pairs = f->size(0);
    r.interleaved = interleaved;
    return true;
}
bool positions_ok(const at::Tensor *t, int64_t tokens, int device) { return kv_indices(t, 1, device) && t->size(0) == tokens; }

int rotary(PyObject **v, PyObject *&result)
{
    apmm_rotation r;
    bool inverse;
    const at::Tensor *x = tensor(v[0]), *at = tensor(v[1]);
    if (!half_type(x) || x->dim() != 3 || !dense_last(*x) || x->get_device() != c10::hip::current_device() || !positions_ok(at, x->size(0), x->get_device()) ||
        !rotation(v[2], v[3], v[4], x->get_device(), r) || !flag(v[5], false, inverse) || x->size(1) > INT32_MAX || x->size(2) > INT32_MAX)
        return 0;
    if (given(v[6])) {
        const at::Tensor *o = tensor(v[6]);
        if (!o || o->scalar_type() != x->scalar_type() || o->get_device() != x->get_device() || o->sizes() != x->sizes() || !dense_last(*o)) return 0;
    }
    Output out;
    if (!output(out, v[6], true, *x, x->sizes(), x->scalar_type())) return result_of(0, out, nullptr, result);
    const at::Tensor &to = *tensor(out.object);
    void *s = stream();
    const bool went = called([&] {
        return lib.rotary(x->size(0), (int)x->size(1), (int)x->size(2), dtype_of(*x), x->data_ptr(), x->stride(0), x->stride(1), static_cast<const int32_t *>(at->data_ptr()), &r, inverse, out.address,
                          to.stride(0), to.stride(1), s);
    });
    return result_of(went ? 1 : -1, out, nullptr, result);
}

int kv_write_rotary(PyObject **v, PyObject *&result)
{
    apmm_kv_cache c;
    apmm_kv_batch b;
    apmm_rotation r;
    const at::Tensor *q = tensor(v[0]), *k = tensor(v[1]), *x = tensor(v[2]);
    if (!q || !k || !x || k->dim() != 3 || q->dim() != 3 || !kv_cache(v[3], v[4], c) || !kv_batch(v[3], v[5], v[6], v[8], k->size(0), b) || q->size(1) > INT32_MAX) return 0;
    const int device = k->get_device();
    if (!kv_rows(q, v[4], q->size(1), c.head_dim, b.tokens) || !kv_rows(k, v[4], c.kv_heads, c.head_dim, b.tokens) || !kv_rows(x, v[4], c.kv_heads, c.head_dim, b.tokens) ||
        !rotation(v[7], v[10], v[11], device, r) || (given(v[9]) && !positions_ok(tensor(v[9]), b.tokens, device)) ||
        (given(v[12]) && !kv_rows(tensor(v[12]), v[4], q->size(1), c.head_dim, b.tokens)))
        return 0;
    const int32_t *at = given(v[9]) ? static_cast<const int32_t *>(tensor(v[9])->data_ptr()) : nullptr;
    Output out;
    if (!output(out, v[12], true, *q, q->sizes(), q->scalar_type())) return result_of(0, out, nullptr, result);
    const at::Tensor &to = *tensor(out.object);
    void *s = stream();
    const bool went = called([&] {
        return lib.kv_write_rotary(&c, &b, (int)q->size(1), at, &r, q->data_ptr(), q->stride(0), q->stride(1), out.address, to.stride(0), to.stride(1), k->data_ptr(), k->stride(0), k->stride(1),
                                   x->data_ptr(), x->stride(0), x->stride(1), s);
    });
    return result_of(went ? 1 : -1, out, nullptr, result);
}

bool kv_weight_rows(const at::Tensor *w, int64_t sequences, int64_t heads, int device)
{
    return w && w->scalar_type() == at::kFloat && w->get_device() == device && w->dim() == 3 && w->size(0) == sequences && w->size(1) == heads && w->size(2) >= 1 && dense_last(*w);
}

int kv_weights(PyObject **v, PyObject *&result)
{
    apmm_kv_cache c;
    apmm_kv_batch b;
    int64_t window = 0, sinks = 0;
    float decay;
    const at::Tensor *q = tensor(v[0]), *w = tensor(v[5]);
    if (!q || q->dim() != 3 || !kv_cache(v[1], v[2], c) || !kv_batch(v[1], v[3], v[4], v[6], q->size(0), b) || q->size(1) > INT32_MAX || !kv_rows(q, v[2], q->size(1), c.head_dim, b.tokens) ||
        !kv_weight_rows(w, b.sequences, c.kv_heads, q->get_device()) || (v[7] && !integer(v[7], -kAny, kAny, window)) || (v[8] && !integer(v[8], -kAny, kAny, sinks)) ||
        (given(v[9]) && !PyFloat_CheckExact(v[9])) || !number(v[10], 1.0, decay) ||
        (given(v[11]) && (!tensor(v[11]) || !tensor(v[11])->is_contiguous() || tensor(v[11])->get_device() != q->get_device())))
        return 0;
    const int heads = (int)q->size(1);
    const float scale = (float)(given(v[9]) ? PyFloat_AS_DOUBLE(v[9]) : 1.0 / std::sqrt((double)c.head_dim));
    const size_t need = given(v[11]) ? 0 : lib.kv_weights_workspace_bytes(&c, &b, heads);
    Output work;
    int done = output(work, v[11], need != 0, *q, {(int64_t)need}, at::kByte);
    if (done) {
        const size_t room = work.address ? bytes(*tensor(work.object)) : 0;
        void *s = stream();
        const bool went = called([&] {
            return lib.kv_weights(&c, &b, heads, q->data_ptr(), q->stride(0), q->stride(1), static_cast<float *>(w->data_ptr()), w->stride(0), w->stride(1), w->size(2), decay, scale, window, sinks,
                                  work.address, room, s);
        });
        done = went ? 1 : -1;
    }
    if (work.made) Py_DECREF(work.object);
    if (done == 1) {
        result = v[5];
        Py_INCREF(result);
    }
    return done;
}

int kv_evict(PyObject **v, PyObject *&result)
{
    apmm_kv_cache c;
    apmm_kv_batch b, to;
    int64_t budget, sinks = 0, recent = 0;
    const at::Tensor *lengths = tensor(v[3]), *w = tensor(v[4]);
    if (!lengths || lengths->dim() != 1 || !kv_cache(v[0], v[1], c) || !kv_batch(v[0], v[2], v[3], nullptr, lengths->size(0), b) || !kv_batch(v[0], v[6], v[3], nullptr, lengths->size(0), to) ||
        !kv_weight_rows(w, b.sequences, c.kv_heads, lengths->get_device()) || !integer(v[5], 1, INT32_MAX, budget) || (v[7] && !integer(v[7], -kAny, kAny, sinks)) ||
        (v[8] && !integer(v[8], -kAny, kAny, recent)))
        return 0;
    const int64_t shape[3] = {b.sequences, c.kv_heads, budget};
    for (int i = 9; i < 12; ++i) {
        if (!given(v[i])) continue;
        const at::Tensor *t = tensor(v[i]);
        if (!t || t->scalar_type() != (i == 10 ? at::kFloat : at::kInt) || t->sizes() != at::IntArrayRef(shape, i == 11 ? 1 : 3) || t->get_device() != lengths->get_device() || !t->is_contiguous())
            return 0;
    }
    if (given(v[12]) && (!tensor(v[12]) || !tensor(v[12])->is_contiguous() || tensor(v[12])->get_device() != lengths->get_device())) return 0;
    const size_t need = given(v[12]) ? 0 : lib.kv_evict_workspace_bytes(&c, b.sequences, b.table_width);
    Output out[3], work;
    int done = output(work, v[12], need != 0, *lengths, {(int64_t)need}, at::kByte);
    for (int i = 0; i < 3 && done; ++i) done = output(out[i], v[9 + i], true, *lengths, at::IntArrayRef(shape, i == 2 ? 1 : 3), i == 1 ? at::kFloat : at::kInt);
    if (done) {
        void *s = stream();
        const bool went = called([&] {
            return lib.kv_evict(&c, b.sequences, b.lengths, b.page_table, b.table_stride, b.table_width, static_cast<const float *>(w->data_ptr()), w->stride(0), w->stride(1), w->size(2), budget, sinks,
                                recent, to.page_table, to.table_stride, to.table_width, static_cast<int32_t *>(out[2].address), static_cast<int32_t *>(out[0].address),
                                static_cast<float *>(out[1].address), work.address, given(v[12]) ? bytes(*tensor(v[12])) : need, s);
        });
        done = went ? 1 : -1;
    }
    if (done == 1) {
        result = PyTuple_Pack(3, out[0].object, out[1].object, out[2].object);
        if (!result) done = -1;
    }
    for (Output &o : out)
        if (o.made) Py_DECREF(o.object);
    if (work.made) Py_DECREF(work.object);
    return done;
}

int w4_gemm(PyObject **v, PyObject *&result)
{
    int64_t N, group;
    const at::Tensor *x = tensor(v[0]), *packed = tensor(v[1]);
    if (!half_type(x) || x->dim() != 2 || !dense_last(*x) || x->get_device() != c10::hip::current_device() || !packed || packed->scalar_type() != at::kByte || packed->get_device() != x->get_device() ||
        !packed->is_contiguous() || !integer(v[2], 0, INT32_MAX, N) || !integer(v[3], 1, INT32_MAX, group))
        return 0;
    const int64_t M = x->size(0), K = x->size(1);
    if (bytes(*packed) < lib.w4_packed_bytes(N, K, (int)group)) return 0;
    if (given(v[4])) {
        const at::Tensor *o = tensor(v[4]);
        if (!o || o->scalar_type() != x->scalar_type() || o->dim() != 2 || o->size(0) != M || o->size(1) != N || o->get_device() != x->get_device() || !dense_last(*o)) return 0;
    }
    if (given(v[5]) && (!tensor(v[5]) || !tensor(v[5])->is_contiguous() || tensor(v[5])->get_device() != x->get_device())) return 0;
    const size_t need = given(v[5]) ? 0 : lib.w4_workspace_bytes(M, N, K, (int)group);
    Output out, work;
    int done = output(out, v[4], true, *x, {M, N}, x->scalar_type()) && output(work, v[5], need != 0, *x, {(int64_t)need}, at::kByte);
    if (done) {
        const at::Tensor &to = *tensor(out.object);
        const size_t room = work.address ? bytes(*tensor(work.object)) : 0;
        void *s = stream();
        const bool went = called([&] {
            return lib.w4_gemm(M, N, K, (int)group, dtype_of(*x), x->data_ptr(), x->stride(0), packed->data_ptr(), out.address, to.stride(0), work.address, room, s);
        });
        done = went ? 1 : -1;
    }
    if (work.made) Py_DECREF(work.object);
    return result_of(done, out, nullptr, result);
}

template <Function F>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t nargs, PyObject *names)
{
    const Signature &s = signatures[F];
    PyObject *v[kMaxArgs], *result = nullptr;
    const int done = end_exceptions(
        [&] {
            if (!place(s, args, nargs, names, v)) return 0;
            return F <= kPackActivations ? pack(F, v, result) : F == kQuantize ? quantize(v, result) : F == kGemm ? gemm(v, result) : F == kFromCodes ? from_codes(v, result) :
                   F == kKvWrite ? kv_write(v, result) : F == kKvRead ? kv_read(v, result) : F == kKvAttention ? kv_attention(v, result) : F == kRotary ? rotary(v, result) :
                   F == kKvWriteRotary ? kv_write_rotary(v, result) : F == kKvWeights ? kv_weights(v, result) : F == kKvEvict ? kv_evict(v, result) : w4_gemm(v, result);
        },
        [] { return 0; });  // (torch's own refusal of a tensor: the general form meets the same one and reports it)
    if (done > 0) return result;
    return done < 0 ? nullptr : general(s, args, nargs, names);
}

// set_library(addresses of the functions in Library's order, _check)
PyObject *set_library(PyObject *, PyObject *args)
{
    unsigned long long at[kLibraryFunctions];
    PyObject *addresses, *fn;
    if (!PyArg_ParseTuple(args, "O!O", &PyTuple_Type, &addresses, &fn)) return nullptr;
    if (PyTuple_GET_SIZE(addresses) != kLibraryFunctions) {
        PyErr_SetString(PyExc_ValueError, "apmm: other functions than this module was built for");
        return nullptr;
    }
    for (int i = 0; i < kLibraryFunctions; ++i) {
        at[i] = PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(addresses, i));
        if (PyErr_Occurred()) return nullptr;
    }
    static_assert(sizeof(lib) == sizeof(at), "addresses of functions alone");
    std::memcpy(&lib, at, sizeof(at));
    Py_INCREF(fn);
    Py_XDECREF(check);
    check = fn;
    loaded = true;
    Py_RETURN_NONE;
}

// set_general(name, function): the Python function of an entry point
PyObject *set_general(PyObject *, PyObject *args)
{
    const char *name;
    PyObject *fn;
    if (!PyArg_ParseTuple(args, "sO", &name, &fn)) return nullptr;
    for (Signature &s : signatures) {
        if (std::strcmp(s.name, name) != 0) continue;
        Py_INCREF(fn);
        Py_XDECREF(s.general);
        s.general = fn;
        Py_RETURN_NONE;
    }
    PyErr_SetString(PyExc_KeyError, name);
    return nullptr;
}

#define ENTRY(F) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(entry<F>)), METH_FASTCALL | METH_KEYWORDS
PyMethodDef methods[] = {
    {"apmm_pack_weights", ENTRY(kPackWeights),
     "apmm_pack_weights(w_codes, q, out=None)\n--\n\nN x K uint8 weight codes -> opaque packed buffer (uint8 tensor)."},
    {"apmm_pack_activations", ENTRY(kPackActivations),
     "apmm_pack_activations(a_codes, p, out=None)\n--\n\nM x K uint8 activation codes -> opaque packed buffer (uint8 tensor)."},
    {"apmm_quantize_pack_activations", ENTRY(kQuantize),
     "apmm_quantize_pack_activations(x_f16, p, out=None, scale_out=None)\n--\n\nM x K float16 activations -> (opaque packed buffer, float16 per-token scales)."},
    {"apmm_gemm", ENTRY(kGemm),
     "apmm_gemm(M, N, K, p, q, a_packed, w_packed, want_i32=True, want_f16=False, w_scale=None, a_scale=None, c_i32=None, c_f16=None, workspace=None, "
     "algo=0)\n--\n\nC = A W^T on packed operands.  Returns (c_i32 or None, c_f16 or None)."},
    {"apmm_gemm_from_codes", ENTRY(kFromCodes),
     "apmm_gemm_from_codes(a_codes, N, p, q, w_packed, want_i32=True, want_f16=False, w_scale=None, a_scale=None, c_i32=None, c_f16=None, "
     "workspace=None)\n--\n\nC = A W^T straight from the M x K uint8 activation codes."},
    {"apmm_kv_write", ENTRY(kKvWrite),
     "apmm_kv_write(k, v, codes, scales, page_table, lengths, starts=None)\n--\n\nQuantise new keys and values (tokens x kv heads x head_dim) into the cache."},
    {"apmm_kv_read", ENTRY(kKvRead),
     "apmm_kv_read(codes, scales, page_table, lengths, tokens, starts=None, k_out=None, v_out=None)\n--\n\nKeys and values of the last tokens of each sequence: (k, v)."},
    {"apmm_kv_attention", ENTRY(kKvAttention),
     "apmm_kv_attention(q, codes, scales, page_table, lengths, starts=None, window=0, sinks=0, scale=None, out=None, workspace=None)\n--\n\n"
     "Causal attention of the new tokens' queries over the cache, which holds their keys and values already."},
    {"apmm_rotary", ENTRY(kRotary),
     "apmm_rotary(x, positions, frequencies, interleaved=False, magnitude=1.0, inverse=False, out=None)\n--\n\n"
     "Turn the pairs of the first 2 * len(frequencies) channels of x by position times frequency."},
    {"apmm_kv_write_rotary", ENTRY(kKvWriteRotary),
     "apmm_kv_write_rotary(q, k, v, codes, scales, page_table, lengths, frequencies, starts=None, positions=None, interleaved=False, magnitude=1.0, q_out=None)\n--\n\n"
     "apmm_rotary of q and k and apmm_kv_write of these k and of v in one launch; the turned q."},
    {"apmm_kv_weights", ENTRY(kKvWeights),
     "apmm_kv_weights(q, codes, scales, page_table, lengths, weights, starts=None, window=0, sinks=0, scale=None, decay=1.0, workspace=None)\n--\n\n"
     "What attention of the new tokens' queries gives each cached token, added to decay * weights."},
    {"apmm_kv_evict", ENTRY(kKvEvict),
     "apmm_kv_evict(codes, scales, page_table, lengths, weights, budget, to_table, sinks=0, recent=0, kept=None, to_weights=None, to_lengths=None, workspace=None)\n--\n\n"
     "Keep of each sequence and head the first tokens, the last and the heaviest others: (places they had, their weights, the new lengths)."},
    {"apmm_w4_gemm", ENTRY(kW4Gemm),
     "apmm_w4_gemm(x, packed, N, group, out=None, workspace=None)\n--\n\nx (M x K, float16 or bfloat16) times packed weights of N channels: M x N of x's type."},
    {"set_library", set_library, METH_VARARGS, nullptr},
    {"set_general", set_general, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "paper_2409_17870_amd._apmm_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject *PyInit__apmm_call()
{
    for (Signature &s : signatures)
        for (int i = 0; i < s.count; ++i)
            if (!(s.keys[i] = PyUnicode_InternFromString(s.args[i]))) return nullptr;
    return PyModule_Create(&module);
}
