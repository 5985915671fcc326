// The Python binding's call path: takes torch tensors apart, allocates outputs, calls the C ABI.
//
// A decode step or a short prefill runs on the GPU for 7 to 15 us, less than what the same steps cost when written in
// Python with ctypes (a dozen attribute reads, the stream object, the conversion of fifteen arguments): there the host
// was the bound.  Here a call costs about a microsecond beside the launches themselves.  The interpreter lock is
// released around the library call, which may block when the launch queue is full.
// Measured through the Python entry points, back to back on one stream (ctypes -> here): one decode step of one sequence
// 9.4 -> 6.5 us, of eight 9.3 -> 8.0, plan and prefill of 1000 tokens in a small geometry 24.2 -> 13.5; the host's share of
// a decode step 10.6 -> 3.4 us.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/cuda/EmptyTensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/bf1.h"

namespace {

PyObject* g_error = nullptr;   // the binding's Bf1Error

struct PyRaised {};            // a Python exception is set

[[noreturn]] void raise(PyObject* type, const char* msg) {
    PyErr_SetString(type, msg);
    throw PyRaised();
}
void require(bool ok, const char* what) {
    if (!ok) raise(PyExc_AssertionError, what);
}
const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) raise(PyExc_TypeError, "expected a torch.Tensor");
    return THPVariable_Unpack(o);
}
long long integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw PyRaised();
    return v;
}
template <typename T>
T* address(PyObject* o) {
    void* p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw PyRaised();
    return static_cast<T*>(p);
}
float scale_of(PyObject* o) {   // None or 0: the library's default
    if (o == Py_None) return 0.f;
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw PyRaised();
    return static_cast<float>(v);
}
void* stream_of(PyObject* o) {  // None: the current stream of the current device
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    return address<void>(o);
}
at::Tensor lse_like(const at::Tensor& q, int64_t heads, int64_t rows) {
    return at::empty({heads, rows}, q.options().dtype(at::kFloat));
}
// One library call with the interpreter lock released; an error status becomes the binding's exception.
template <typename F>
void call(F&& f) {
    int rc;
    {
        PyThreadState* state = PyEval_SaveThread();
        rc = f();
        PyEval_RestoreThread(state);
    }
    if (rc == BF1_OK) return;
    PyObject* e = PyObject_CallFunction(g_error, "is", rc, bf1_last_error());
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    throw PyRaised();
}
PyObject* pair(const at::Tensor& a, const at::Tensor& b) {
    PyObject *x = THPVariable_Wrap(a), *y = THPVariable_Wrap(b);
    PyObject* t = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return t;
}

// Where a call runs: on the device of its tensors, on `stream` or, if that is None, on the device's current stream; what it
// allocates belongs to that stream.
struct Place {
    c10::cuda::CUDAGuard device;
    c10::cuda::OptionalCUDAStreamGuard guard;
    void* stream;
    Place(const at::Tensor& t, PyObject* o) : device((require(t.is_cuda(), "the tensors have to be on a CUDA device"), t.device())) {
        if (o == Py_None) {
            stream = c10::cuda::getCurrentCUDAStream(t.device().index()).stream();
        } else {
            stream = address<void>(o);
            guard.reset_stream(c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(stream), t.device().index()));
        }
    }
};
// A new tensor on the current device's current stream, without a way through the dispatcher.
at::Tensor fresh(at::IntArrayRef sizes, const at::Tensor& like, at::ScalarType type) {
    return at::detail::empty_cuda(sizes, type, like.device(), std::nullopt);
}
// A part of `flat`'s memory as a contiguous tensor of its own.
at::Tensor part_of(const at::Tensor& flat, int64_t offset, at::IntArrayRef sizes) {
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(flat.storage()), flat.key_set(), flat.dtype());
    t.unsafeGetTensorImpl()->set_storage_offset(offset);
    t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
    return t;
}
// [tokens, heads, d] bf16 with the dimensions of a head side by side, on `like`'s device
bf1_rows rows_of(const at::Tensor& t, const at::Tensor& like, const char* what) {
    require(t.device() == like.device() && t.scalar_type() == at::kBFloat16 && t.dim() == 3 && (t.size(2) == 1 || t.stride(2) == 1), what);
    return {t.data_ptr(), t.size(0) > 1 ? t.stride(0) : 0, t.size(1) > 1 ? t.stride(1) : 0};
}
// The same for a result: its rows and heads each have a place of their own.
bf1_rows result_rows(const at::Tensor& t, const at::Tensor& like, const char* what) {
    require((t.size(0) < 2 || t.stride(0) != 0) && (t.size(1) < 2 || t.stride(1) != 0), "an output's rows must not share memory");
    return rows_of(t, like, what);
}
template <typename T>
T* array_of(const at::Tensor& t, const at::Tensor& like, at::ScalarType type, const char* what) {
    require(t.device() == like.device() && t.scalar_type() == type && t.is_contiguous(), what);
    return static_cast<T*>(t.data_ptr());
}

struct Qkv {
    int64_t T, hq, hkv, d;
};
Qkv check_qkv(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v) {
    for (const at::Tensor* t : {&q, &k, &v})
        require(t->is_cuda() && t->scalar_type() == at::kBFloat16 && t->is_contiguous() && t->dim() == 3,
                "q, k and v must be contiguous 3-d bf16 CUDA tensors");
    require(k.sizes() == v.sizes() && k.size(0) == q.size(0) && k.size(2) == q.size(2), "shapes of q, k and v do not match");
    return {q.size(0), q.size(1), k.size(1), q.size(2)};
}

// Every function takes positional arguments; `*`-marked ones may be None.
// plan_route(cu_seqlens, total, max_seqlen, cfg address, route address, stream*)
PyObject* plan_route(PyObject* const* a) {
    const at::Tensor& cu = tensor(a[0]);
    require(cu.is_cuda() && cu.scalar_type() == at::kInt && cu.is_contiguous(), "cu_seqlens must be a contiguous int32 CUDA tensor");
    const int32_t batch = static_cast<int32_t>(cu.numel() - 1), max_seqlen = static_cast<int32_t>(integer(a[2]));
    const int64_t total = integer(a[1]);
    const auto* cfg = address<const bf1_route_cfg>(a[3]);
    const auto* route = address<const bf1_route>(a[4]);
    void* stream = stream_of(a[5]);
    const auto* cup = static_cast<const int32_t*>(cu.data_ptr());
    call([&] { return bf1_plan_route(cup, batch, total, max_seqlen, cfg, route, stream); });
    Py_RETURN_NONE;
}

// forward(which, q, k, v, cu_seqlens, max_seqlen, scale*, out*, lse*, stream*, x, y, z)
//   which 0: bf1_attn_fwd, x = route address;  1: bf1_dense_causal_fwd, x = work tensor*;
//   2: bf1_attn_fwd_noalloc, x = total tokens, y = cfg address, z = status tensor*
PyObject* forward(PyObject* const* a) {
    const long long which = integer(a[0]);
    const at::Tensor &q = tensor(a[1]), &k = tensor(a[2]), &v = tensor(a[3]), &cu = tensor(a[4]);
    const Qkv g = check_qkv(q, k, v);
    const int32_t max_seqlen = static_cast<int32_t>(integer(a[5]));
    const float scale = scale_of(a[6]);
    const at::Tensor out = a[7] == Py_None ? at::empty_like(q) : tensor(a[7]);
    const at::Tensor lse = a[8] == Py_None ? lse_like(q, g.hq, g.T) : tensor(a[8]);
    void* stream = stream_of(a[9]);
    const void *qp = q.data_ptr(), *kp = k.data_ptr(), *vp = v.data_ptr();
    const auto* cup = static_cast<const int32_t*>(cu.data_ptr());
    const int32_t batch = static_cast<int32_t>(cu.numel() - 1), hq = g.hq, hkv = g.hkv, d = g.d;
    void* op = out.data_ptr();
    auto* lp = static_cast<float*>(lse.data_ptr());
    if (which == 0) {
        const auto* route = address<const bf1_route>(a[10]);
        call([&] { return bf1_attn_fwd(qp, kp, vp, cup, batch, g.T, max_seqlen, hq, hkv, d, scale, route, op, lp, stream); });
    } else if (which == 1) {
        auto* work = a[10] == Py_None ? nullptr : static_cast<int32_t*>(tensor(a[10]).data_ptr());
        call([&] { return bf1_dense_causal_fwd(qp, kp, vp, cup, batch, g.T, max_seqlen, hq, hkv, d, scale, op, lp, work, stream); });
    } else {
        const int64_t total = a[10] == Py_None ? g.T : integer(a[10]);
        const auto* cfg = address<const bf1_route_cfg>(a[11]);
        auto* status = a[12] == Py_None ? nullptr : static_cast<int32_t*>(tensor(a[12]).data_ptr());
        call([&] {
            return bf1_attn_fwd_noalloc(qp, kp, vp, cup, batch, total, max_seqlen, hq, hkv, d, scale, cfg, op, lp, status, stream);
        });
    }
    return pair(out, lse);
}

// backward(q, k, v, o, lse, d_o, cu_seqlens, max_seqlen, route address, scale*, workspace, stream*)
PyObject* backward(PyObject* const* a) {
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]), &o = tensor(a[3]), &lse = tensor(a[4]),
                     &d_o = tensor(a[5]), &cu = tensor(a[6]), &ws = tensor(a[10]);
    const Qkv g = check_qkv(q, k, v);
    require(d_o.sizes() == q.sizes() && d_o.scalar_type() == at::kBFloat16 && d_o.is_contiguous(),
            "d_o must be a contiguous bf16 tensor of q's shape");
    const int32_t max_seqlen = static_cast<int32_t>(integer(a[7]));
    const auto* route = address<const bf1_route>(a[8]);
    const float scale = scale_of(a[9]);
    void* stream = stream_of(a[11]);
    const at::Tensor dq = at::empty_like(q), dk = at::empty_like(k), dv = at::empty_like(v);
    const int32_t batch = static_cast<int32_t>(cu.numel() - 1);
    const void *qp = q.data_ptr(), *kp = k.data_ptr(), *vp = v.data_ptr(), *op = o.data_ptr(), *gp = d_o.data_ptr();
    const auto* lp = static_cast<const float*>(lse.data_ptr());
    const auto* cup = static_cast<const int32_t*>(cu.data_ptr());
    void *wp = ws.data_ptr(), *dqp = dq.data_ptr(), *dkp = dk.data_ptr(), *dvp = dv.data_ptr();
    call([&] {
        return bf1_attn_bwd(qp, kp, vp, op, lp, gp, cup, batch, g.T, max_seqlen, static_cast<int32_t>(g.hq),
                            static_cast<int32_t>(g.hkv), static_cast<int32_t>(g.d), scale, route, wp, dqp, dkp, dvp, stream);
    });
    PyObject *x = THPVariable_Wrap(dq), *y = THPVariable_Wrap(dk), *z = THPVariable_Wrap(dv);
    PyObject* t = x && y && z ? PyTuple_Pack(3, x, y, z) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    Py_XDECREF(z);
    return t;
}

// plan_decode(seqlens, page_table, cfg address, plan address, stream*)
PyObject* plan_decode(PyObject* const* a) {
    const at::Tensor &seqlens = tensor(a[0]), &table = tensor(a[1]);
    require(seqlens.is_cuda() && seqlens.scalar_type() == at::kInt && table.scalar_type() == at::kInt && table.dim() == 2,
            "seqlens and the 2-d page_table must be int32 CUDA tensors");
    const auto* cfg = address<const bf1_route_cfg>(a[2]);
    const auto* plan = address<const bf1_decode_plan>(a[3]);
    void* stream = stream_of(a[4]);
    const int32_t batch = static_cast<int32_t>(table.size(0)), pages = static_cast<int32_t>(table.size(1));
    const auto *sp = static_cast<const int32_t*>(seqlens.data_ptr()), *tp = static_cast<const int32_t*>(table.data_ptr());
    call([&] { return bf1_plan_decode(sp, tp, pages, batch, cfg, plan, stream); });
    Py_RETURN_NONE;
}

// decode(q, k_pages, v_pages, seqlens, plan address, workspace, scale*, out*, lse*, stream*)
PyObject* decode(PyObject* const* a) {
    const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]), &seqlens = tensor(a[3]), &ws = tensor(a[5]);
    require(q.dim() == 3 && k.dim() == 4 && k.size(1) == 64 && k.size(3) == q.size(2) && v.sizes() == k.sizes(),
            "q must be [batch, hq, d], k_pages and v_pages [pages, 64, hkv, d]");
    const auto* plan = address<const bf1_decode_plan>(a[4]);
    const float scale = scale_of(a[6]);
    const at::Tensor out = a[7] == Py_None ? at::empty_like(q) : tensor(a[7]);
    const at::Tensor lse = a[8] == Py_None ? lse_like(q, q.size(1), q.size(0)) : tensor(a[8]);
    void* stream = stream_of(a[9]);
    const int32_t batch = q.size(0), hq = q.size(1), d = q.size(2), pages = k.size(0), hkv = k.size(2);
    const void *qp = q.data_ptr(), *kp = k.data_ptr(), *vp = v.data_ptr();
    const auto* sp = static_cast<const int32_t*>(seqlens.data_ptr());
    void *wp = ws.data_ptr(), *op = out.data_ptr();
    auto* lp = static_cast<float*>(lse.data_ptr());
    call([&] { return bf1_decode_fwd(qp, kp, vp, pages, sp, batch, hq, hkv, d, scale, plan, wp, op, lp, stream); });
    return pair(out, lse);
}

// The table of a rope has to lie where the call runs.
void check_table(const at::Tensor& turns, const at::Tensor& like) {
    array_of<const double>(turns, like, at::kDouble, "the rope's table must be on the device of the tensors");
}

// decode_fp8(q, k_pages, v_pages, k_scales, v_scales, seqlens, plan address, its counts, workspace, scale*, out*, lse*, stream*, cu_tokens*)
PyObject* decode_fp8(PyObject* const* a) {
    const at::Tensor &q = tensor(a[0]), &kp = tensor(a[1]), &vp = tensor(a[2]), &ks = tensor(a[3]), &vs = tensor(a[4]), &seqlens = tensor(a[5]),
                     &count = tensor(a[7]), &ws = tensor(a[8]);
    const Place place(q, a[12]);
    const void* qp = array_of<const void>(q, q, at::kBFloat16, "q must be a contiguous bf16 tensor");
    const char* const what = "k_pages and v_pages must be contiguous float8_e4m3fn tensors [pages, 64, hkv, d] on the device of q";
    const void *kpp = array_of<const void>(kp, q, at::kFloat8_e4m3fn, what), *vpp = array_of<const void>(vp, q, at::kFloat8_e4m3fn, what);
    require(q.dim() == 3 && kp.dim() == 4 && kp.size(1) == 64 && kp.size(3) == q.size(2) && vp.sizes() == kp.sizes() && kp.size(0) <= INT32_MAX, what);
    const char* const scales = "k_scales and v_scales must be contiguous fp32 tensors [pages, hkv] on the device of q";
    const auto *ksp = array_of<const float>(ks, q, at::kFloat, scales), *vsp = array_of<const float>(vs, q, at::kFloat, scales);
    require(ks.dim() == 2 && ks.size(0) == kp.size(0) && ks.size(1) == kp.size(2) && vs.sizes() == ks.sizes(), scales);
    const auto* sp = array_of<const int32_t>(seqlens, q, at::kInt, "seqlens must be a contiguous int32 tensor on the device of q");
    array_of<int32_t>(count, q, at::kInt, "the plan must be on the device of the tensors");
    const int32_t* cu = nullptr;
    if (a[13] != Py_None) {
        const at::Tensor& t = tensor(a[13]);
        cu = array_of<const int32_t>(t, q, at::kInt, "cu_tokens must be a contiguous int32 tensor on the device of q");
        require(seqlens.dim() == 1 && seqlens.size(0) == count.size(0) && t.dim() == 1 && t.size(0) == count.size(0) + 1,
                "seqlens and the plan must be of the same batch, cu_tokens [batch + 1]");
        require(q.size(0) <= INT32_MAX, "too many rows");
    } else {
        require(seqlens.dim() == 1 && seqlens.size(0) == q.size(0) && count.size(0) == q.size(0), "q, seqlens and the plan must be of the same batch");
    }
    const auto* plan = address<const bf1_decode_plan>(a[6]);
    const float scale = scale_of(a[9]);
    const int32_t rows = q.size(0), batch = seqlens.size(0), hq = q.size(1), d = q.size(2), pages = kp.size(0), hkv = kp.size(2);
    void* wp = array_of<void>(ws, q, at::kByte, "the workspace must be a byte tensor on the device of q");
    require(ws.numel() >= bf1_decode_fp8_workspace_bytes(batch, hq, hkv, plan->max_degree, d), "the workspace is too small: see decode_fp8_workspace");
    const at::Tensor out = a[10] == Py_None ? at::empty(q.sizes(), q.options()) : tensor(a[10]);
    const at::Tensor lse = a[11] == Py_None ? lse_like(q, hq, rows) : tensor(a[11]);
    require(out.sizes() == q.sizes() && lse.dim() == 2 && lse.size(0) == hq && lse.size(1) == rows, "out must have the shape of q, lse must be [hq, rows of q]");
    void* op = array_of<void>(out, q, at::kBFloat16, "out must be a contiguous bf16 tensor on the device of q");
    auto* lp = array_of<float>(lse, q, at::kFloat, "lse must be a contiguous fp32 tensor on the device of q");
    if (batch > 0 && rows > 0 && cu)
        call([&] { return bf1_decode_fwd_fp8_packed(qp, rows, cu, kpp, vpp, ksp, vsp, pages, sp, batch, hq, hkv, d, scale, plan, wp, op, lp, place.stream); });
    else if (batch > 0 && rows > 0)
        call([&] { return bf1_decode_fwd_fp8(qp, kpp, vpp, ksp, vsp, pages, sp, batch, hq, hkv, d, scale, plan, wp, op, lp, place.stream); });
    return pair(out, lse);
}

// rope(backward, q, k*, positions, rope address, its table, out_q*, out_k*, stream*)
PyObject* rope(PyObject* const* a) {
    const bool back = integer(a[0]) != 0, keys = a[2] != Py_None;
    const at::Tensor &q = tensor(a[1]), &k = keys ? tensor(a[2]) : q, &pos = tensor(a[3]);
    const auto* table = address<const bf1_rope>(a[4]);
    const char* const what = "q, k and their outputs must be 3-d bf16 tensors on one CUDA device, the last dimension contiguous";
    require(keys || a[7] == Py_None, "out_k is given without k");
    const Place place(q, a[8]);
    check_table(tensor(a[5]), q);
    const bf1_rows qr = rows_of(q, q, what), kr = rows_of(k, q, what);
    require(k.size(0) == q.size(0) && k.size(2) == q.size(2), "q and k must have the same tokens and head dimension");
    const auto* pp = array_of<const int32_t>(pos, q, at::kInt, "positions must be a contiguous int32 tensor on the same device");
    require(pos.dim() == 1 && pos.size(0) == q.size(0), "positions must have an entry for every token");
    at::Tensor out_q, out_k;
    if (keys && a[6] == Py_None && a[7] == Py_None) {    // both in one piece of memory: a second allocation would cost as much as the kernel's launch
        const at::Tensor flat = fresh({q.numel() + k.numel()}, q, at::kBFloat16);
        out_q = part_of(flat, 0, q.sizes());
        out_k = part_of(flat, q.numel(), k.sizes());
    } else {
        out_q = a[6] == Py_None ? fresh(q.sizes(), q, at::kBFloat16) : tensor(a[6]);
        out_k = !keys ? out_q : a[7] == Py_None ? fresh(k.sizes(), q, at::kBFloat16) : tensor(a[7]);
    }
    require(out_q.sizes() == q.sizes() && out_k.sizes() == (keys ? k : q).sizes(), "the outputs must have the shapes of q and k");
    const bf1_rows oq = result_rows(out_q, q, what), ok = result_rows(out_k, q, what);
    const int32_t tokens = q.size(0), hq = q.size(1), hkv = keys ? k.size(1) : 0, d = q.size(2);
    call([&] {
        return back ? bf1_rope_bwd(&qr, &kr, pp, tokens, hq, hkv, d, table, &oq, &ok, place.stream)
                    : bf1_rope_fwd(&qr, &kr, pp, tokens, hq, hkv, d, table, &oq, &ok, place.stream);
    });
    if (keys) return pair(out_q, out_k);
    PyObject* x = THPVariable_Wrap(out_q);
    PyObject* t = x ? PyTuple_Pack(2, x, Py_None) : nullptr;
    Py_XDECREF(x);
    return t;
}

// plan_cache(seqlens, new_lens, page_table, num_pages, free_pages*, free_count*, plan address, its status, seqlens_out, free_count_out, stream*)
PyObject* plan_cache(PyObject* const* a) {
    const at::Tensor &lens = tensor(a[0]), &add = tensor(a[1]), &table = tensor(a[2]);
    const Place place(lens, a[10]);
    const char* const what = "plan_cache: contiguous int32 tensors on one CUDA device";
    const auto *lp = array_of<const int32_t>(lens, lens, at::kInt, what), *np = array_of<const int32_t>(add, lens, at::kInt, what);
    auto* tp = array_of<int32_t>(table, lens, at::kInt, what);
    array_of<int32_t>(tensor(a[7]), lens, at::kInt, "the plan must be on the device of the tensors");
    bf1_cache_plan plan = *address<const bf1_cache_plan>(a[6]);
    const long long num_pages = integer(a[3]);
    require(num_pages >= 1 && num_pages <= INT32_MAX, "num_pages out of range");
    require(lens.dim() == 1 && lens.size(0) == plan.batch && add.sizes() == lens.sizes() && table.dim() == 2 && table.size(0) == plan.batch,
            "seqlens and new_lens must be [batch], page_table [batch, pages], batch the plan's");
    require((a[4] == Py_None) == (a[5] == Py_None), "free_pages and free_count go together");
    int32_t* fp = nullptr;
    const int32_t* cp = nullptr;
    if (a[4] != Py_None) {
        const at::Tensor &pages = tensor(a[4]), &count = tensor(a[5]);
        fp = array_of<int32_t>(pages, lens, at::kInt, what);
        cp = array_of<const int32_t>(count, lens, at::kInt, what);
        require(pages.numel() >= num_pages && count.numel() == 1, "free_pages must have room for num_pages, free_count must be one number");
    }
    const at::Tensor &lens_out = tensor(a[8]), &count_out = tensor(a[9]);
    require(lens_out.sizes() == lens.sizes() && count_out.numel() == 1, "seqlens_out must be [batch], free_count_out one number");
    if (plan.batch > 0) plan.seqlens = array_of<int32_t>(lens_out, lens, at::kInt, what);
    plan.free_count = array_of<int32_t>(count_out, lens, at::kInt, what);
    const int32_t width = static_cast<int32_t>(table.size(1));
    call([&] { return bf1_plan_cache(lp, np, tp, width, static_cast<int32_t>(num_pages), fp, cp, &plan, place.stream); });
    Py_RETURN_NONE;
}

// cache_write(k, v, k_pages, v_pages, plan address, its status, k_scales*, v_scales*, rope address*, its table*, q*, out_q*, stream*)
PyObject* cache_write(PyObject* const* a) {
    const at::Tensor &k = tensor(a[0]), &v = tensor(a[1]), &kp = tensor(a[2]), &vp = tensor(a[3]);
    const bool queries = a[10] != Py_None;
    require(queries || a[11] == Py_None, "out_q is given without q");
    const Place place(k, a[12]);
    const char* const what = "k, v, q and out_q must be 3-d bf16 tensors on one CUDA device, the last dimension contiguous";
    const bf1_rows kr = rows_of(k, k, what), vr = rows_of(v, k, what);
    require(v.sizes() == k.sizes(), "k and v must have the same shape");
    const auto* plan = address<const bf1_cache_plan>(a[4]);
    array_of<int32_t>(tensor(a[5]), k, at::kInt, "the plan must be on the device of the tensors");
    const bool scaled = a[6] != Py_None;
    require(scaled == (a[7] != Py_None), "k_scales and v_scales go together");
    const at::ScalarType type = scaled ? at::kFloat8_e4m3fn : at::kBFloat16;
    for (const at::Tensor* t : {&kp, &vp}) {
        array_of<void>(*t, k, type, scaled ? "with scales the pages must be contiguous float8_e4m3fn tensors" : "without scales the pages must be contiguous bf16 tensors");
        require(t->dim() == 4 && t->size(1) == 64 && t->size(2) == k.size(1) && t->size(3) == k.size(2) && t->size(0) == kp.size(0) && t->size(0) <= INT32_MAX,
                "k_pages and v_pages must be [pages, 64, hkv, d]");
    }
    float* scales[2] = {nullptr, nullptr};
    for (int i = 0; scaled && i < 2; ++i) {
        const at::Tensor& t = tensor(a[6 + i]);
        scales[i] = array_of<float>(t, k, at::kFloat, "k_scales and v_scales must be contiguous fp32 tensors");
        require(t.dim() == 2 && t.size(0) == kp.size(0) && t.size(1) == k.size(1), "k_scales and v_scales must be [pages, hkv]");
    }
    const bf1_rope* rope = nullptr;
    if (a[8] != Py_None) {
        rope = address<const bf1_rope>(a[8]);
        check_table(tensor(a[9]), k);
    }
    bf1_rows qr = {}, oq = {};
    at::Tensor out_q;
    int32_t hq = 0;
    if (queries) {
        const at::Tensor& q = tensor(a[10]);
        qr = rows_of(q, k, what);
        require(q.size(0) == k.size(0) && q.size(2) == k.size(2), "q and k must have the same tokens and head dimension");
        out_q = a[11] == Py_None ? at::empty(q.sizes(), q.options()) : tensor(a[11]);
        require(out_q.sizes() == q.sizes(), "out_q must have the shape of q");
        oq = result_rows(out_q, k, what);
        hq = q.size(1);
    }
    const int32_t tokens = k.size(0), hkv = k.size(1), d = k.size(2), pages = kp.size(0);
    void *kpp = kp.data_ptr(), *vpp = vp.data_ptr();
    call([&] { return bf1_cache_write(&kr, &vr, &qr, tokens, hq, hkv, d, plan, rope, pages, kpp, vpp, scales[0], scales[1], &oq, place.stream); });
    if (queries) return THPVariable_Wrap(out_q);
    Py_RETURN_NONE;
}

// Argument count, C++ and torch exceptions.
template <PyObject* (*F)(PyObject* const*), int kArgs>
PyObject* entry(PyObject*, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != kArgs) {
        PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", kArgs, n);
        return nullptr;
    }
    try {
        return F(args);
    } catch (const PyRaised&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

PyObject* set_error(PyObject*, PyObject* type) {
    Py_INCREF(type);
    Py_XDECREF(g_error);
    g_error = type;
    Py_RETURN_NONE;
}

#define BF1_ENTRY(name, args) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<name, args>)), METH_FASTCALL, nullptr}
PyMethodDef g_methods[] = {
    {"set_error", set_error, METH_O, nullptr},
    BF1_ENTRY(plan_route, 6),
    BF1_ENTRY(forward, 13),
    BF1_ENTRY(backward, 12),
    BF1_ENTRY(plan_decode, 5),
    BF1_ENTRY(decode, 10),
    BF1_ENTRY(decode_fp8, 14),
    BF1_ENTRY(rope, 9),
    BF1_ENTRY(plan_cache, 11),
    BF1_ENTRY(cache_write, 13),
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_host", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host() { return PyModule_Create(&g_module); }
