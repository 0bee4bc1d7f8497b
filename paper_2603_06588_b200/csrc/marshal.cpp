// Argument marshalling of the short calls (rotary append, logit edits, cache pages) for binding.py: checks the tensors, fills the
// C structs and calls the C ABI.  These calls take a few microseconds on the device, and reading some twenty tensors' types, shapes
// and strides from Python takes longer than that: hook_rope_append on one row takes 11.7 us through ctypes and struct.pack and
// 5.4 us from here, with a launch of 2.9 us in it.
//
// Nothing is computed here.  A failed check raises AssertionError, like the checks of the other calls; a code of the library is
// returned as an int, which binding.py turns into its exception.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstdint>
#include <utility>
#include <vector>

#include "hook_attn.h"

namespace {

constexpr int kPage = 16;                        // tokens of a page

struct Refused {
    const char* why;
};
struct Raised {};                                // a Python error is set

void check(bool ok, const char* why)
{
    if (!ok) throw Refused{why};
}

int32_t narrow(int64_t x, const char* why = "a size beyond 32 bits")
{
    check(x >= INT32_MIN && x <= INT32_MAX, why);
    return (int32_t)x;
}

int64_t integer(PyObject* x)
{
    const long long v = PyLong_AsLongLong(x);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
}

// The arguments of a call: the entry point's address, the handle, its device, the stream (None: the current one), then its own.
struct Call {
    PyObject* const* args;
    Py_ssize_t count, next = 4;
    hook_attn_handle* handle;
    int device;
    cudaStream_t stream;

    Call(PyObject* const* a, Py_ssize_t n, Py_ssize_t want) : args(a), count(n)
    {
        check(n == want, "number of arguments");
        handle = reinterpret_cast<hook_attn_handle*>(integer(a[1]));
        device = (int)integer(a[2]);
        stream = a[3] == Py_None ? current() : reinterpret_cast<cudaStream_t>(integer(a[3]));
    }
    cudaStream_t current() const { return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream(); }
    template <typename F>
    F* entry() const { return reinterpret_cast<F*>(integer(args[0])); }
    PyObject* other() { return args[next++]; }

    const at::Tensor* maybe(const char* what)
    {
        PyObject* x = other();
        if (x == Py_None) return nullptr;
        check(THPVariable_Check(x), what);
        const at::Tensor& t = THPVariable_Unpack(x);
        check(t.is_cuda() && t.get_device() == device, "a tensor is not on the handle's device");
        return &t;
    }
    const at::Tensor& tensor(const char* what, int64_t dims)
    {
        const at::Tensor* t = maybe(what);
        check(t && t->dim() == dims, what);
        return *t;
    }
    // One dimension of a known length, without gaps; `length` -1: any.
    const at::Tensor* maybe_list(const char* what, at::ScalarType type, int64_t length)
    {
        const at::Tensor* t = maybe(what);
        if (t) check(t->scalar_type() == type && t->dim() == 1 && t->is_contiguous() && (length < 0 || t->size(0) == length), what);
        return t;
    }
    const at::Tensor& list(const char* what, at::ScalarType type, int64_t length)
    {
        const at::Tensor* t = maybe_list(what, type, length);
        check(t, what);
        return *t;
    }
    int32_t* status()
    {
        const at::Tensor* t = maybe("status");
        if (t) check(t->scalar_type() == at::kInt && t->numel() > 0, "status: int32 [1]");
        return pointer<int32_t>(t);
    }

    template <typename T>
    static T* pointer(const at::Tensor* t) { return t ? static_cast<T*>(t->data_ptr()) : nullptr; }

    // Memory for a result: taken in the order of the stream that the call goes to, so that neither what used it before nor what gets
    // it afterwards is still to run, or already running, there.
    at::Tensor make(at::IntArrayRef shape, at::ScalarType type) const
    {
        const auto options = at::TensorOptions().dtype(type).device(at::kCUDA, (c10::DeviceIndex)device);
        if (stream == current()) return at::empty(shape, options);
        const auto index = (c10::DeviceIndex)device;
        c10::cuda::CUDAStreamGuard guard(stream ? c10::cuda::getStreamFromExternal(stream, index) : c10::cuda::getDefaultCUDAStream(index));
        return at::empty(shape, options);
    }
    template <typename F, typename... A>
    int issue(A... a) const
    {
        F* f = entry<F>();
        int rc;
        Py_BEGIN_ALLOW_THREADS rc = f(handle, a..., static_cast<void*>(stream));
        Py_END_ALLOW_THREADS return rc;
    }
};

// Runs a call's body; what it throws becomes a Python error.
template <typename Body>
PyObject* guarded(Body body)
{
    try {
        return body();
    } catch (const Refused& r) {
        PyErr_SetString(PyExc_AssertionError, r.why);
    } catch (const Raised&) {
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error");
    }
    return nullptr;
}

PyObject* result(int rc, at::Tensor t) { return rc == HOOK_ATTN_OK ? THPVariable_Wrap(std::move(t)) : PyLong_FromLong(rc); }

int32_t dtype_of(const at::Tensor& t)
{
    switch (t.scalar_type()) {
        case at::kBFloat16: return HOOK_DTYPE_BF16;
        case at::kHalf: return HOOK_DTYPE_F16;
        case at::kFloat: return HOOK_DTYPE_F32;
        default: throw Refused{"bf16, fp16 or fp32"};
    }
}

PyObject* rope_append(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        Call c(args, n, 4 + 16);
        hook_rope_params p = {};
        const at::Tensor &q = c.tensor("q [T, Hq, D]", 3), &k = c.tensor("k [T, Hkv, D]", 3), &v = c.tensor("v [T, Hkv, D]", 3);
        const at::Tensor &kc = c.tensor("k_cache [pages, 16, Hkv, D]", 4), &vc = c.tensor("v_cache [pages, 16, Hkv, D]", 4);
        const at::Tensor &table = c.tensor("block_table [seqs, pages]", 2), &lens = c.list("seq_lens: int32 [seqs]", at::kInt, table.size(0));
        const at::Tensor& freq = c.list("inv_freq: fp32 [R / 2]", at::kFloat, -1);
        const int64_t rows = q.size(0), pairs = freq.size(0);
        const at::Tensor *cu = c.maybe_list("cu_q_lens: int32 [seqs + 1]", at::kInt, table.size(0) + 1), *positions = c.maybe("positions");
        PyObject* sections = c.other();
        p.axis_order = narrow(integer(c.other()));
        p.pairing = narrow(integer(c.other()));
        p.factor = (float)PyFloat_AsDouble(c.other());
        if (PyErr_Occurred()) throw Raised{};
        const at::Tensor* given = c.maybe("q_out");
        p.status = c.status();

        check(k.sizes() == v.sizes() && k.size(0) == rows && k.size(2) == q.size(2), "k and v [T, Hkv, D]");
        check(k.scalar_type() == q.scalar_type() && v.scalar_type() == q.scalar_type(), "q, k and v of one type");
        check(rows == 0 || (q.stride(2) == 1 && k.stride(2) == 1 && v.stride(2) == 1), "q, k and v: neighbouring elements of a head");
        check(kc.sizes() == vc.sizes() && kc.strides() == vc.strides() && kc.stride(3) == 1 && kc.size(3) == q.size(2) && kc.size(2) == k.size(1),
              "k_cache and v_cache [pages, 16, Hkv, D] with the same strides");
        check(kc.scalar_type() == at::kBFloat16 && vc.scalar_type() == at::kBFloat16, "a bf16 cache");
        check(table.scalar_type() == at::kInt && table.is_contiguous(), "block_table: int32, contiguous");
        p.num_axes = 1;
        p.axis_pairs[0] = narrow(pairs);
        if (sections != Py_None) {
            PyObject* seq = PySequence_Fast(sections, "axis_pairs");
            if (!seq) throw Raised{};
            const Py_ssize_t axes = PySequence_Fast_GET_SIZE(seq);
            int64_t each[HOOK_ROPE_MAX_AXES] = {};
            for (Py_ssize_t i = 0; i < axes && i < HOOK_ROPE_MAX_AXES && !PyErr_Occurred(); ++i) each[i] = PyLong_AsLongLong(PySequence_Fast_GET_ITEM(seq, i));
            Py_DECREF(seq);
            if (PyErr_Occurred()) throw Raised{};
            check(axes >= 1 && axes <= HOOK_ROPE_MAX_AXES, "1 to 4 axes");
            p.num_axes = (int32_t)axes;
            for (int i = 0; i < axes; ++i) p.axis_pairs[i] = narrow(each[i]);
        }
        if (positions) {
            check(positions->scalar_type() == at::kInt && positions->dim() == 2 && positions->size(0) == p.num_axes && positions->size(1) == rows &&
                      (rows <= 1 || positions->stride(1) == 1), "positions: int32 [axes, T]");
            p.position_axis_stride = positions->stride(0);
        }
        if (given) check(given->scalar_type() == at::kBFloat16 && given->sizes() == q.sizes() && given->is_contiguous(), "q_out: bf16, contiguous, like q");
        at::Tensor out = given ? *given : c.make(q.sizes(), at::kBFloat16);

        p.num_seqs = narrow(table.size(0));
        p.total_q = narrow(rows);
        p.num_q_heads = narrow(q.size(1));
        p.num_kv_heads = narrow(k.size(1));
        p.head_dim = narrow(q.size(2));
        p.page_size = narrow(kc.size(1));
        p.num_blocks = narrow(kc.size(0));
        p.max_blocks_per_seq = narrow(table.size(1));
        p.dtype = dtype_of(q);
        p.rotary_dim = narrow(2 * pairs);
        p.q = q.data_ptr();
        p.k = k.data_ptr();
        p.v = v.data_ptr();
        p.q_row_stride = q.stride(0);
        p.q_head_stride = q.stride(1);
        p.k_row_stride = k.stride(0);
        p.k_head_stride = k.stride(1);
        p.v_row_stride = v.stride(0);
        p.v_head_stride = v.stride(1);
        p.inv_freq = Call::pointer<float>(&freq);
        p.positions = Call::pointer<int32_t>(positions);
        p.q_out = out.data_ptr();
        p.k_cache = kc.data_ptr();
        p.v_cache = vc.data_ptr();
        p.kv_block_stride = kc.stride(0);
        p.kv_token_stride = kc.stride(1);
        p.kv_head_stride = kc.stride(2);
        p.block_table = Call::pointer<int32_t>(&table);
        p.seq_lens = Call::pointer<int32_t>(&lens);
        p.cu_q_lens = Call::pointer<int32_t>(cu);
        return result(c.issue<decltype(hook_rope_append)>(&p), std::move(out));
    });
}

PyObject* adjust_logits(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        Call c(args, n, 4 + 14);
        hook_logits_params p = {};
        const at::Tensor& logits = c.tensor("logits [rows, vocab]", 2);
        const at::Tensor* given = c.maybe("out");
        const at::Tensor& out = given ? *given : logits;
        const int64_t rows = logits.size(0), vocab = logits.size(1);
        const at::Tensor* tokens = c.maybe("tokens");
        const at::Tensor *prompt = c.maybe_list("prompt_lens: int32 [rows]", at::kInt, rows), *total = c.maybe_list("total_lens: int32 [rows]", at::kInt, rows);
        const at::Tensor *repetition = c.maybe_list("repetition: fp32 [rows]", at::kFloat, rows), *presence = c.maybe_list("presence: fp32 [rows]", at::kFloat, rows);
        const at::Tensor* frequency = c.maybe_list("frequency: fp32 [rows]", at::kFloat, rows);
        const at::Tensor* offsets = c.maybe_list("bias_offsets: int32 [rows + 1]", at::kInt, rows + 1);
        const at::Tensor *named = c.maybe_list("bias_tokens: int32", at::kInt, -1), *values = c.maybe_list("bias_values: fp32", at::kFloat, -1);
        const at::Tensor* mask = c.maybe("mask");
        const at::Tensor* mask_rows = c.maybe_list("mask_rows: int32 [rows]", at::kInt, rows);
        p.status = c.status();

        check(out.sizes() == logits.sizes() && (vocab == 1 || (logits.stride(1) == 1 && out.stride(1) == 1)), "logits and out [rows, vocab]");
        check(rows <= 1 || (logits.stride(0) >= vocab && out.stride(0) >= vocab), "rows of logits that do not overlap");
        p.num_rows = narrow(rows);
        p.vocab_size = narrow(vocab);
        p.dtype = dtype_of(logits);
        p.out_dtype = dtype_of(out);
        p.logits = logits.data_ptr();
        p.out = out.data_ptr();
        p.logits_row_stride = std::max(logits.stride(0), vocab);
        p.out_row_stride = std::max(out.stride(0), vocab);
        if (tokens) {
            check(tokens->scalar_type() == at::kInt && tokens->dim() == 2 && tokens->size(0) == rows && (tokens->size(1) <= 1 || tokens->stride(1) == 1),
                  "tokens: int32 [rows, max_tokens]");
            check(prompt && total, "prompt_lens and total_lens with tokens");
            p.max_tokens = narrow(tokens->size(1));
            p.tokens_row_stride = tokens->stride(0);
            // a buffer without room has no address, but lengths that are checked: any address stands for it, none of it is read
            p.tokens = tokens->size(1) > 0 ? Call::pointer<int32_t>(tokens) : Call::pointer<int32_t>(total);
            p.prompt_lens = Call::pointer<int32_t>(prompt);
            p.total_lens = Call::pointer<int32_t>(total);
        }
        p.repetition = Call::pointer<float>(repetition);
        p.presence = Call::pointer<float>(presence);
        p.frequency = Call::pointer<float>(frequency);
        if (offsets) {
            check(named && values && named->size(0) == values->size(0), "bias_tokens and bias_values of one length with bias_offsets");
            p.num_bias = narrow(named->size(0));
            p.bias_offsets = Call::pointer<int32_t>(offsets);
            p.bias_tokens = Call::pointer<int32_t>(named);
            p.bias_values = Call::pointer<float>(values);
        }
        if (mask) {
            check((mask->scalar_type() == at::kInt || mask->scalar_type() == at::kUInt32) && mask->dim() == 2 && 32 * mask->size(1) >= vocab &&
                      (mask->size(1) == 1 || mask->stride(1) == 1), "mask: int32 [masks, ceil(vocab / 32)]");
            p.num_masks = narrow(mask->size(0));
            p.mask_row_stride = mask->stride(0);
            p.mask = Call::pointer<uint32_t>(mask);
            p.mask_rows = Call::pointer<int32_t>(mask_rows);
        }
        return result(c.issue<decltype(hook_adjust_logits)>(&p), out);
    });
}

// The four arguments that every call on a pool has: block_table, seq_lens, page_refs, status.
hook_cache_pool pool_of(Call& c, const at::Tensor** table = nullptr)
{
    hook_cache_pool p = {};
    const at::Tensor &t = c.tensor("block_table [seqs, pages]", 2), &lens = c.list("seq_lens: int32 [seqs]", at::kInt, t.size(0));
    const at::Tensor& refs = c.list("page_refs: int32 [pages]", at::kInt, -1);
    check(t.scalar_type() == at::kInt && t.is_contiguous(), "block_table: int32, contiguous");
    p.num_seqs = narrow(t.size(0));
    p.max_blocks_per_seq = narrow(t.size(1));
    p.num_blocks = narrow(refs.size(0));
    p.page_size = kPage;
    p.block_table = Call::pointer<int32_t>(&t);
    p.seq_lens = Call::pointer<int32_t>(&lens);
    p.page_refs = Call::pointer<int32_t>(&refs);
    p.status = c.status();
    if (table) *table = &t;
    return p;
}

PyObject* cache_fork(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        Call c(args, n, 4 + 6);
        const hook_cache_pool p = pool_of(c);
        const at::Tensor& parents = c.list("parents: int32", at::kInt, -1);
        const at::Tensor& children = c.list("children: int32, one for each parent", at::kInt, parents.size(0));
        return PyLong_FromLong(c.issue<decltype(hook_cache_fork)>(&p, Call::pointer<const int32_t>(&parents), Call::pointer<const int32_t>(&children),
                                                                  narrow(parents.size(0))));
    });
}

PyObject* cache_extend(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        Call c(args, n, 4 + 6);
        const hook_cache_pool p = pool_of(c);
        const at::Tensor& rows = c.list("new_rows: int32 [seqs]", at::kInt, p.num_seqs);
        const at::Tensor* given = c.maybe("pairs");
        if (given) check(given->scalar_type() == at::kInt && given->is_contiguous() && given->dim() == 2 && given->size(0) == p.num_seqs && given->size(1) == 2,
                         "pairs: int32 [seqs, 2]");
        at::Tensor pairs = given ? *given : c.make({p.num_seqs, 2}, at::kInt);
        const int rc = c.issue<decltype(hook_cache_extend)>(&p, Call::pointer<const int32_t>(&rows), Call::pointer<int32_t>(&pairs));
        return result(rc, std::move(pairs));
    });
}

PyObject* cache_free(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        Call c(args, n, 4 + 6);
        const hook_cache_pool p = pool_of(c);
        const at::Tensor& seqs = c.list("seqs: int32", at::kInt, -1);
        const at::Tensor* keep = c.maybe_list("keep_lens: int32, one for each sequence", at::kInt, seqs.size(0));
        return PyLong_FromLong(c.issue<decltype(hook_cache_free)>(&p, Call::pointer<const int32_t>(&seqs), Call::pointer<const int32_t>(keep),
                                                                  narrow(seqs.size(0))));
    });
}

PyObject* cache_compact(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        Call c(args, n, 4 + 4);
        const at::Tensor* table;
        const hook_cache_pool p = pool_of(c, &table);
        at::Tensor out[5] = {c.make(table->sizes(), at::kInt), c.make({p.num_blocks}, at::kInt), c.make({p.num_blocks}, at::kInt),
                             c.make({p.num_blocks / 2, 2}, at::kInt), c.make({1}, at::kInt)};
        int32_t* at[5];
        for (int i = 0; i < 5; ++i) at[i] = Call::pointer<int32_t>(&out[i]);
        const int rc = c.issue<decltype(hook_cache_compact)>(&p, at[0], at[1], at[2], at[3], at[4]);
        if (rc != HOOK_ATTN_OK) return PyLong_FromLong(rc);
        PyObject* all = PyTuple_New(5);
        for (int i = 0; all && i < 5; ++i) {
            PyObject* x = THPVariable_Wrap(std::move(out[i]));
            if (!x) {
                Py_DECREF(all);
                return nullptr;
            }
            PyTuple_SET_ITEM(all, i, x);
        }
        return all;
    });
}

PyObject* cache_copy_pages(PyObject*, PyObject* const* args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject* {
        Call c(args, n, 4 + 4);
        hook_cache_copy_params p = {};
        PyObject* caches = PySequence_Fast(c.other(), "a list of (k_cache, v_cache)");
        if (!caches) throw Raised{};
        struct Held {
            PyObject* x;
            ~Held() { Py_DECREF(x); }
        } held{caches};
        const Py_ssize_t layers = PySequence_Fast_GET_SIZE(caches);
        std::vector<void*> at[2];
        const at::Tensor* first = nullptr;
        for (Py_ssize_t l = 0; l < layers; ++l) {
            PyObject* pair = PySequence_Fast_GET_ITEM(caches, l);
            check((PyTuple_Check(pair) || PyList_Check(pair)) && PySequence_Fast_GET_SIZE(pair) == 2, "a list of (k_cache, v_cache)");
            for (int i = 0; i < 2; ++i) {
                PyObject* x = PySequence_Fast_GET_ITEM(pair, i);
                check(THPVariable_Check(x), "a list of (k_cache, v_cache)");
                const at::Tensor& t = THPVariable_Unpack(x);
                if (!first) first = &t;
                check(t.dim() == 4 && t.sizes() == first->sizes() && t.strides() == first->strides() && t.stride(3) == 1 && t.scalar_type() == at::kBFloat16,
                      "caches of one shape and one set of strides, bf16 [pages, 16, Hkv, D]");
                check(t.is_cuda() && t.get_device() == c.device, "a tensor is not on the handle's device");
                at[i].push_back(t.data_ptr());
            }
        }
        const at::Tensor& pairs = c.tensor("pairs [n, 2]", 2);
        const at::Tensor* count = c.maybe("num_pairs");
        p.status = c.status();
        check(pairs.scalar_type() == at::kInt && pairs.size(1) == 2 && pairs.is_contiguous(), "pairs: int32 [n, 2], contiguous");
        if (count) check(count->scalar_type() == at::kInt && count->numel() == 1, "num_pairs: int32 [1]");
        if (!first) return PyLong_FromLong(HOOK_ATTN_OK);
        p.num_layers = narrow(layers);
        p.num_blocks = narrow(first->size(0));
        p.page_size = narrow(first->size(1));
        p.num_kv_heads = narrow(first->size(2));
        p.head_dim = narrow(first->size(3));
        p.max_pairs = narrow(pairs.size(0));
        p.kv_block_stride = first->stride(0);
        p.kv_token_stride = first->stride(1);
        p.kv_head_stride = first->stride(2);
        p.k_caches = at[0].data();
        p.v_caches = at[1].data();
        p.pairs = Call::pointer<int32_t>(&pairs);
        p.num_pairs = Call::pointer<int32_t>(count);
        return PyLong_FromLong(c.issue<decltype(hook_cache_copy_pages)>(&p));
    });
}

#define CALL(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {CALL(rope_append), CALL(adjust_logits), CALL(cache_fork), CALL(cache_extend), CALL(cache_free), CALL(cache_compact),
                         CALL(cache_copy_pages), {nullptr, nullptr, 0, nullptr}};
PyModuleDef definition = {PyModuleDef_HEAD_INIT, "_marshal", "Argument marshalling of the short calls of libhook_attn.so.", -1, methods,
                          nullptr, nullptr, nullptr, nullptr};

// This file reads tensors by the layout of the torch and the Python that it was compiled for: with others it is not loaded.
bool made_for_these()
{
    PyObject* torch = Py_Version >> 16 == PY_VERSION_HEX >> 16 ? PyImport_ImportModule("torch") : nullptr;
    PyObject* version = torch ? PyObject_GetAttrString(torch, "__version__") : nullptr;
    Py_XDECREF(torch);
    const bool same = version && PyUnicode_Check(version) && PyUnicode_CompareWithASCIIString(version, HOOK_TORCH_VERSION) == 0;
    if (!PyErr_Occurred() && !same)
        PyErr_Format(PyExc_ImportError, "_marshal.so was built for torch %s and Python %d.%d", HOOK_TORCH_VERSION, PY_MAJOR_VERSION, PY_MINOR_VERSION);
    Py_XDECREF(version);
    return same;
}

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return made_for_these() ? PyModule_Create(&definition) : nullptr; }
