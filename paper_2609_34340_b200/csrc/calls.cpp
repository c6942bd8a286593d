// The binding's frequent calls, from Python objects straight to the C ABI.
//
// A ctypes call of one of these functions spends 10 to 15 us on the host: a Python object per pointer, tensor slices for
// matrix b of a plan, a parameter struct, a Stream object.  The kernels of a decode step take 3 to 9 us, so that was the
// time of the call.  Here tensors are unpacked in C++ (about 1 us in all).  Arguments and error codes are those of the C
// ABI; checks that concern Python arguments raise AssertionError as the Python wrappers do.
#include <Python.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "variopath.h"

namespace {

struct Failed {};                       // a Python error has been set

[[noreturn]] void fail(PyObject* type, const char* text) {
    if (!PyErr_Occurred()) PyErr_SetString(type, text);
    throw Failed{};
}

const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) fail(PyExc_TypeError, "a tensor is expected");
    return THPVariable_Unpack(o);
}
void* ptr(PyObject* o) { return o == Py_None ? nullptr : tensor(o).data_ptr(); }

long long integer(PyObject* o) {
    if (PyLong_CheckExact(o)) {
        const long long v = PyLong_AsLongLong(o);
        if (v == -1 && PyErr_Occurred()) throw Failed{};
        return v;
    }
    PyObject* n = PyNumber_Long(o);
    if (!n) throw Failed{};
    const long long v = PyLong_AsLongLong(n);
    Py_DECREF(n);
    if (v == -1 && PyErr_Occurred()) throw Failed{};
    return v;
}

struct Ref {                            // an owned reference
    PyObject* o;
    explicit Ref(PyObject* p) : o(p) { if (!o) throw Failed{}; }
    ~Ref() { Py_DECREF(o); }
    Ref(const Ref&) = delete;
};

#define NAMES(X) X(_h) X(value) X(N) X(lambda_ns) X(granule_bytes) X(k_target) X(n_start) X(i_aa) X(k_max) X(n_steps) X(chan_id) \
    X(lane_dst) X(lane_inst) X(lane_bytes) X(send_off) X(recv_off) X(tau_ns) X(status) X(cuda_stream) \
    X(experts) X(topk) X(scoring) X(n_group) X(topk_group) X(group_top) X(renormalise) X(scale)
#define DECLARE(n) PyObject* s_##n;
NAMES(DECLARE)

long long attr_int(PyObject* o, PyObject* name) { Ref r(PyObject_GetAttr(o, name)); return integer(r.o); }
void* attr_ptr(PyObject* o, PyObject* name) { Ref r(PyObject_GetAttr(o, name)); return ptr(r.o); }

// Address of row b of a plan array (its first dimension is the batch).
template <typename T>
T* row_of(PyObject* plan, PyObject* name, long long b, long long* last = nullptr) {
    Ref r(PyObject_GetAttr(plan, name));
    const at::Tensor& t = tensor(r.o);
    if (b < 0) b += t.size(0);
    if (b < 0 || b >= t.size(0)) fail(PyExc_IndexError, "matrix index out of range");
    if (last) *last = t.size(t.dim() - 1);
    return (T*)((char*)t.data_ptr() + b * t.stride(0) * (long long)t.element_size());
}

void* stream_of(PyObject* o) {
    if (o == Py_None) return (void*)c10::cuda::getCurrentCUDAStream().stream();
    Ref r(PyObject_GetAttr(o, s_cuda_stream));
    return (void*)(uintptr_t)(unsigned long long)integer(r.o);
}

const vp_catalog* handle_of(PyObject* catalog) {
    Ref h(PyObject_GetAttr(catalog, s__h));
    if (h.o == Py_None) return nullptr;
    Ref v(PyObject_GetAttr(h.o, s_value));
    return v.o == Py_None ? nullptr : (const vp_catalog*)PyLong_AsVoidPtr(v.o);
}

vp_sched_params params_of(PyObject* p, long long N) {
    vp_sched_params q;
    q.lambda_ns = attr_int(p, s_lambda_ns);
    q.granule_bytes = attr_int(p, s_granule_bytes);
    q.k_target = (int32_t)attr_int(p, s_k_target);
    q.n_start = (int32_t)attr_int(p, s_n_start);
    q.i_aa = (int32_t)attr_int(p, s_i_aa);
    const long long k = attr_int(p, s_k_max);
    q.k_max = (int32_t)(k ? k : 8 * N);
    return q;
}

size_t bytes_of(const at::Tensor& t) { return (size_t)t.numel() * t.element_size(); }
bool is_i32(const at::Tensor& t) { return t.is_cuda() && t.scalar_type() == at::kInt && t.is_contiguous(); }
bool on_gpu(const at::Tensor& t) { return t.is_cuda() && t.is_contiguous(); }
void check(bool ok, const char* text) { if (!ok) fail(PyExc_AssertionError, text); }

template <typename F>
PyObject* call(Py_ssize_t n, Py_ssize_t want, F f) {
    if (n != want) { PyErr_SetString(PyExc_TypeError, "wrong number of arguments"); return nullptr; }
    try {
        return PyLong_FromLong(f());
    } catch (const Failed&) {
    } catch (const std::exception& e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
#define WITHOUT_GIL(rc, expr) { Py_BEGIN_ALLOW_THREADS rc = (expr); Py_END_ALLOW_THREADS }

// ---- one function per call; argument order as in binding.py ------------------------------------------------------------

using SchedFn = int (*)(const vp_catalog*, const vp_sched_params*, const int64_t*, const int64_t*, int, int32_t*, int32_t*, int16_t*,
                        uint16_t*, int64_t*, int64_t*, int64_t*, int64_t*, int32_t*, void*, size_t, void*);

// (catalog, params, demand, tau_ns_in, plan, workspace, stream)
int schedule(SchedFn fn, PyObject* const* a, bool host) {
    const at::Tensor& demand = tensor(a[2]);
    check((host ? !demand.is_cuda() : demand.is_cuda()) && demand.scalar_type() == at::kLong && demand.is_contiguous(),
          host ? "demand: a contiguous int64 host tensor" : "demand: a contiguous int64 device tensor");
    const long long N = attr_int(a[0], s_N), B = demand.size(0);
    check(host || (demand.dim() == 3 && demand.size(1) == N && demand.size(2) == N), "demand: [B, N, N]");
    const vp_catalog* c = handle_of(a[0]);
    const vp_sched_params p = params_of(a[1], N);
    PyObject* plan = a[4];
    void *n_steps = attr_ptr(plan, s_n_steps), *chan = attr_ptr(plan, s_chan_id), *dst = attr_ptr(plan, s_lane_dst),
         *inst = attr_ptr(plan, s_lane_inst), *bytes = attr_ptr(plan, s_lane_bytes), *so = attr_ptr(plan, s_send_off),
         *ro = attr_ptr(plan, s_recv_off), *tau = attr_ptr(plan, s_tau_ns), *st = attr_ptr(plan, s_status);
    const at::Tensor& ws = tensor(a[5]);
    const int64_t *d = (const int64_t*)demand.data_ptr(), *tin = (const int64_t*)ptr(a[3]);
    void *w = ws.data_ptr(), *stream = stream_of(a[6]);
    const size_t wb = (size_t)ws.numel();
    int rc;
    WITHOUT_GIL(rc, fn(c, &p, d, tin, (int)B, (int32_t*)n_steps, (int32_t*)chan, (int16_t*)dst, (uint16_t*)inst, (int64_t*)bytes,
                       (int64_t*)so, (int64_t*)ro, (int64_t*)tau, (int32_t*)st, w, wb, stream))
    return rc;
}
PyObject* schedule_batch(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 7, [&] { return schedule(vp_schedule_batch, a, false); });
}
PyObject* schedule_batch_host(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 7, [&] { return schedule(vp_schedule_batch_host, a, true); });
}
PyObject* schedule_batch_host_used(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 7, [&] { return schedule(vp_schedule_batch_host_used, a, true); });
}

// (expert_idx, experts_per_rank, N, row_bytes, src0, out, status, stream)
PyObject* demand_from_routing(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 8, [&] {
        const at::Tensor& idx = tensor(a[0]);
        check(is_i32(idx) && idx.dim() == 3, "expert_idx: a contiguous int32 device tensor [n_src, T, topk]");
        const int epr = (int)integer(a[1]), N = (int)integer(a[2]), src0 = (int)integer(a[4]);
        const int64_t rb = integer(a[3]);
        void *out = ptr(a[5]), *st = ptr(a[6]), *stream = stream_of(a[7]);
        int rc;
        WITHOUT_GIL(rc, vp_demand_from_routing((const int32_t*)idx.data_ptr(), (int)idx.size(0), (int)idx.size(1), (int)idx.size(2), epr, N,
                                               src0, rb, (int64_t*)out, (int32_t*)st, stream))
        return rc;
    });
}

// (plan, b, rank, expert_idx, experts_per_rank, rows, staged, src_map, status, workspace or None for the static form, stream)
PyObject* pack(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 11, [&] {
        const at::Tensor &idx = tensor(a[3]), &rows = tensor(a[5]), &staged = tensor(a[6]);
        check(is_i32(idx), "expert_idx: a contiguous int32 device tensor");
        check(on_gpu(rows) && on_gpu(staged), "rows, staged: contiguous device tensors");
        check(idx.dim() == 2 && rows.dim() >= 2, "expert_idx: [T, topk], rows: [T, H]");
        const long long b = integer(a[1]);
        long long N;
        const int32_t* n_steps = row_of<int32_t>(a[0], s_n_steps, b);
        const int16_t* dst = row_of<int16_t>(a[0], s_lane_dst, b, &N);
        const int64_t *bytes = row_of<int64_t>(a[0], s_lane_bytes, b), *so = row_of<int64_t>(a[0], s_send_off, b);
        const int rank = (int)integer(a[2]), k_max = (int)attr_int(a[0], s_k_max), epr = (int)integer(a[4]);
        const int64_t rb = rows.size(1) * (int64_t)rows.element_size(), cap = (int64_t)bytes_of(staged);
        void *map = ptr(a[7]), *st = ptr(a[8]), *stream = stream_of(a[10]);
        const bool own = a[9] != Py_None;
        void* ws = own ? tensor(a[9]).data_ptr() : nullptr;
        const size_t wb = own ? (size_t)tensor(a[9]).numel() : 0;
        int rc;
        WITHOUT_GIL(rc, own ? vp_pack(n_steps, dst, bytes, so, (int)N, rank, k_max, (const int32_t*)idx.data_ptr(), (int)idx.size(0),
                                      (int)idx.size(1), epr, rows.data_ptr(), rb, staged.data_ptr(), cap, (int32_t*)map, (int32_t*)st, ws, wb, stream)
                            : vp_pack_static(n_steps, dst, bytes, so, (int)N, rank, k_max, (const int32_t*)idx.data_ptr(), (int)idx.size(0),
                                             (int)idx.size(1), epr, rows.data_ptr(), rb, staged.data_ptr(), cap, (int32_t*)map, (int32_t*)st, stream))
        return rc;
    });
}

// (plan, b, rank, staged, recv_bufs, recv_capacity, arrived, status, stream)
PyObject* exchange_put(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 9, [&] {
        const long long b = integer(a[1]);
        long long N;
        const int32_t* n_steps = row_of<int32_t>(a[0], s_n_steps, b);
        const int16_t* dst = row_of<int16_t>(a[0], s_lane_dst, b, &N);
        const int64_t *so = row_of<int64_t>(a[0], s_send_off, b), *ro = row_of<int64_t>(a[0], s_recv_off, b);
        const int rank = (int)integer(a[2]), k_max = (int)attr_int(a[0], s_k_max);
        void *staged = ptr(a[3]), *bufs = ptr(a[4]), *cap = ptr(a[5]), *arrived = ptr(a[6]), *st = ptr(a[7]), *stream = stream_of(a[8]);
        int rc;
        WITHOUT_GIL(rc, vp_exchange_put(n_steps, dst, so, ro, (int)N, rank, k_max, staged, (void* const*)bufs, (const int64_t*)cap,
                                        (uint64_t* const*)arrived, (int32_t*)st, stream))
        return rc;
    });
}

// (plan, b, rank, recv, recv_expert, experts_per_rank, out, expert_off, out_src, out_map, status, workspace, stream)
PyObject* unpack(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 13, [&] {
        const at::Tensor &recv = tensor(a[3]), &ex = tensor(a[4]), &out = tensor(a[6]), &ws = tensor(a[11]);
        check(on_gpu(recv) && recv.dim() == 2 && on_gpu(out), "recv, out: contiguous device tensors, recv [capacity_rows, H]");
        check(is_i32(ex), "recv_expert: a contiguous int32 device tensor");
        check(ex.numel() >= recv.size(0) && bytes_of(out) >= bytes_of(recv), "recv_expert, out: as large as recv");
        const long long b = integer(a[1]);
        long long N;
        const int32_t* n_steps = row_of<int32_t>(a[0], s_n_steps, b);
        const int16_t* dst = row_of<int16_t>(a[0], s_lane_dst, b, &N);
        const int64_t* ro = row_of<int64_t>(a[0], s_recv_off, b);
        const int rank = (int)integer(a[2]), k_max = (int)attr_int(a[0], s_k_max), epr = (int)integer(a[5]);
        const int64_t rb = recv.size(1) * (int64_t)recv.element_size();
        void *off = ptr(a[7]), *src = ptr(a[8]), *map = ptr(a[9]), *st = ptr(a[10]), *stream = stream_of(a[12]);
        int rc;
        WITHOUT_GIL(rc, vp_unpack(n_steps, dst, ro, (int)N, rank, k_max, recv.data_ptr(), rb, recv.size(0), (const int32_t*)ex.data_ptr(), epr,
                                  out.data_ptr(), (int32_t*)off, (int32_t*)src, (int32_t*)map, (int32_t*)st, ws.data_ptr(), (size_t)ws.numel(), stream))
        return rc;
    });
}

// (plan, b, rank, expert_idx, experts_per_rank, recv, out, out_map, status, workspace, stream)
PyObject* unpack_tokens(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 11, [&] {
        const at::Tensor &idx = tensor(a[3]), &recv = tensor(a[5]), &out = tensor(a[6]), &ws = tensor(a[9]);
        check(is_i32(idx) && idx.dim() == 2, "expert_idx: a contiguous int32 device tensor [T, topk]");
        check(on_gpu(recv) && recv.dim() == 2 && on_gpu(out), "recv, out: contiguous device tensors, recv [capacity_rows, H]");
        const int64_t rb = recv.size(1) * (int64_t)recv.element_size();
        check((int64_t)bytes_of(out) >= idx.numel() * rb, "out: a row per routed copy");
        const long long b = integer(a[1]);
        long long N;
        const int32_t* n_steps = row_of<int32_t>(a[0], s_n_steps, b);
        const int16_t* dst = row_of<int16_t>(a[0], s_lane_dst, b, &N);
        const int64_t *bytes = row_of<int64_t>(a[0], s_lane_bytes, b), *ro = row_of<int64_t>(a[0], s_recv_off, b);
        const int rank = (int)integer(a[2]), k_max = (int)attr_int(a[0], s_k_max), epr = (int)integer(a[4]);
        void *map = ptr(a[7]), *st = ptr(a[8]), *stream = stream_of(a[10]);
        int rc;
        WITHOUT_GIL(rc, vp_unpack_tokens(n_steps, dst, bytes, ro, (int)N, rank, k_max, (const int32_t*)idx.data_ptr(), (int)idx.size(0),
                                         (int)idx.size(1), epr, recv.data_ptr(), rb, recv.size(0), out.data_ptr(), (int32_t*)map, (int32_t*)st,
                                         ws.data_ptr(), (size_t)ws.numel(), stream))
        return rc;
    });
}

// ---- the operators around the AlltoAllv: tensors on one device, whose current stream is the default ------------------------

struct Device {                         // that device, current for the call
    c10::Device d;
    c10::cuda::CUDAGuard guard;
    explicit Device(const at::Tensor& t) : d(first(t)), guard(d) {}
    static c10::Device first(const at::Tensor& t) {
        check(t.is_cuda(), "a device tensor is expected");
        return t.device();
    }
    const at::Tensor& has(const at::Tensor& t) const {
        check(t.device() == d, "tensors on one device are expected");
        return t;
    }
    void* stream(PyObject* o) const {
        return o == Py_None ? (void*)c10::cuda::getCurrentCUDAStream(d.index()).stream() : stream_of(o);
    }
};

int type_of(const at::Tensor& t) {
    const auto s = t.scalar_type();
    check(s == at::kBFloat16 || s == at::kHalf || s == at::kFloat, "bfloat16, float16 or float32 is expected");
    return s == at::kBFloat16 ? VP_BF16 : (s == at::kHalf ? VP_F16 : VP_F32);
}
// Elements from one row to the next of a matrix whose rows are contiguous and do not overlap.
int64_t row_stride(const at::Tensor& t, const char* text) {
    check(t.dim() == 2 && (t.size(1) <= 1 || t.stride(1) == 1) && (t.size(0) <= 1 || t.stride(0) >= t.size(1)), text);
    return t.size(0) <= 1 ? t.size(1) : t.stride(0);
}
bool is_matrix(const at::Tensor& t, at::ScalarType s, int64_t rows, int64_t cols) {
    return t.scalar_type() == s && t.is_contiguous() && t.dim() == 2 && t.size(0) == rows && t.size(1) == cols;
}
int int_size(int64_t n) {
    check(n < ((int64_t)1 << 31), "fewer than 2^31 rows are expected");
    return (int)n;
}

vp_route_params route_params_of(PyObject* p) {
    vp_route_params q;
    q.experts = (int32_t)attr_int(p, s_experts);
    q.topk = (int32_t)attr_int(p, s_topk);
    Ref scoring(PyObject_GetAttr(p, s_scoring));
    const bool text = PyUnicode_Check(scoring.o);
    const bool softmax = text && PyUnicode_CompareWithASCIIString(scoring.o, "softmax") == 0;
    check(softmax || (text && PyUnicode_CompareWithASCIIString(scoring.o, "sigmoid") == 0), "scoring: \"softmax\" or \"sigmoid\"");
    q.scoring = softmax ? VP_SCORE_SOFTMAX : VP_SCORE_SIGMOID;
    q.n_group = (int32_t)attr_int(p, s_n_group);
    q.topk_group = (int32_t)attr_int(p, s_topk_group);
    q.group_top = (int32_t)attr_int(p, s_group_top);
    q.renormalise = attr_int(p, s_renormalise) != 0;
    Ref scale(PyObject_GetAttr(p, s_scale));
    q.scale = (float)PyFloat_AsDouble(scale.o);
    if (PyErr_Occurred()) throw Failed{};
    return q;
}

// (params, logits, bias, expert_idx, weights, stream)
PyObject* route(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 6, [&] {
        const vp_route_params p = route_params_of(a[0]);
        const at::Tensor& z = tensor(a[1]);
        const Device dev(z);
        const at::Tensor &idx = dev.has(tensor(a[3])), &w = dev.has(tensor(a[4]));
        const int64_t ld = row_stride(z, "logits: [T, experts], rows contiguous");
        check(z.size(1) == p.experts, "logits: [T, experts]");
        check(is_matrix(idx, at::kInt, z.size(0), p.topk) && is_matrix(w, at::kFloat, z.size(0), p.topk),
              "expert_idx, weights: contiguous int32 and float32 [T, topk]");
        const void* bias = nullptr;
        if (a[2] != Py_None) {
            const at::Tensor& b = dev.has(tensor(a[2]));
            check(b.scalar_type() == at::kFloat && b.is_contiguous() && b.numel() == p.experts, "bias: contiguous float32 [experts]");
            bias = b.data_ptr();
        }
        const int type = type_of(z), T = int_size(z.size(0));
        void* stream = dev.stream(a[5]);
        int rc;
        WITHOUT_GIL(rc, vp_route(&p, z.data_ptr(), type, ld, T, (const float*)bias, (int32_t*)idx.data_ptr(), (float*)w.data_ptr(), stream))
        return rc;
    });
}

// (params, logits, expert_idx, grad_weights, grad_logits, stream)
PyObject* route_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 6, [&] {
        const vp_route_params p = route_params_of(a[0]);
        const at::Tensor& z = tensor(a[1]);
        const Device dev(z);
        const at::Tensor &idx = dev.has(tensor(a[2])), &g = dev.has(tensor(a[3])), &out = dev.has(tensor(a[4]));
        const int64_t ld = row_stride(z, "logits: [T, experts], rows contiguous"), out_ld = row_stride(out, "grad_logits: [T, experts], rows contiguous");
        check(z.size(1) == p.experts && out.sizes() == z.sizes() && out.scalar_type() == z.scalar_type(),
              "logits, grad_logits: [T, experts] of one type");
        check(is_matrix(idx, at::kInt, z.size(0), p.topk) && is_matrix(g, at::kFloat, z.size(0), p.topk),
              "expert_idx, grad_weights: contiguous int32 and float32 [T, topk]");
        const int type = type_of(z), T = int_size(z.size(0));
        void* stream = dev.stream(a[5]);
        int rc;
        WITHOUT_GIL(rc, vp_route_backward(&p, z.data_ptr(), type, ld, T, (const int32_t*)idx.data_ptr(), (const float*)g.data_ptr(),
                                          out.data_ptr(), out_ld, stream))
        return rc;
    });
}

// (rows, expert_idx, weights, base, out, stream)
PyObject* combine(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 6, [&] {
        const at::Tensor& rows = tensor(a[0]);
        const Device dev(rows);
        const at::Tensor &idx = dev.has(tensor(a[1])), &w = dev.has(tensor(a[2])), &out = dev.has(tensor(a[4]));
        check(idx.dim() == 2 && is_matrix(idx, at::kInt, idx.size(0), idx.size(1)) && is_matrix(w, at::kFloat, idx.size(0), idx.size(1)),
              "expert_idx, weights: contiguous int32 and float32 [T, topk]");
        const int64_t T = idx.size(0), topk = idx.size(1);
        check(rows.dim() == 2 && is_matrix(rows, rows.scalar_type(), T * topk, rows.size(1)), "rows: contiguous [T * topk, H]");
        check(is_matrix(out, rows.scalar_type(), T, rows.size(1)), "out: contiguous [T, H] of the rows' type");
        const void* base = nullptr;
        if (a[3] != Py_None) {
            const at::Tensor& b = dev.has(tensor(a[3]));
            check(is_matrix(b, rows.scalar_type(), T, rows.size(1)), "base: contiguous [T, H] of the rows' type");
            base = b.data_ptr();
        }
        const int type = type_of(rows), t = int_size(T), k = int_size(topk);
        void* stream = dev.stream(a[5]);
        int rc;
        WITHOUT_GIL(rc, vp_combine(rows.data_ptr(), type, (const int32_t*)idx.data_ptr(), (const float*)w.data_ptr(), t, k, rows.size(1), base,
                                   out.data_ptr(), stream))
        return rc;
    });
}

// (grad, rows, expert_idx, weights, grad_rows or None, grad_weights or None, stream)
PyObject* combine_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 7, [&] {
        const at::Tensor& grad = tensor(a[0]);
        const Device dev(grad);
        const at::Tensor &idx = dev.has(tensor(a[2])), &w = dev.has(tensor(a[3]));
        check(idx.dim() == 2 && is_matrix(idx, at::kInt, idx.size(0), idx.size(1)) && is_matrix(w, at::kFloat, idx.size(0), idx.size(1)),
              "expert_idx, weights: contiguous int32 and float32 [T, topk]");
        const int64_t T = idx.size(0), topk = idx.size(1);
        check(grad.dim() == 2 && is_matrix(grad, grad.scalar_type(), T, grad.size(1)), "grad: contiguous [T, H]");
        const auto many = [&](PyObject* o, const char* text) -> void* {
            if (o == Py_None) return nullptr;
            const at::Tensor& t = dev.has(tensor(o));
            check(is_matrix(t, grad.scalar_type(), T * topk, grad.size(1)), text);
            return t.data_ptr();
        };
        void *rows = many(a[1], "rows: contiguous [T * topk, H] of the gradient's type"),
             *grad_rows = many(a[4], "grad_rows: contiguous [T * topk, H] of the gradient's type"), *grad_weights = nullptr;
        if (a[5] != Py_None) {
            const at::Tensor& g = dev.has(tensor(a[5]));
            check(is_matrix(g, at::kFloat, T, topk), "grad_weights: contiguous float32 [T, topk]");
            grad_weights = g.data_ptr();
        }
        const int type = type_of(grad), t = int_size(T), k = int_size(topk);
        void* stream = dev.stream(a[6]);
        int rc;
        WITHOUT_GIL(rc, vp_combine_backward(grad.data_ptr(), rows, type, (const int32_t*)idx.data_ptr(), (const float*)w.data_ptr(), t, k,
                                            grad.size(1), grad_rows, (float*)grad_weights, stream))
        return rc;
    });
}

const int32_t* count_of(const Device& dev, PyObject* o) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = dev.has(tensor(o));
    check(t.scalar_type() == at::kInt && t.numel() == 1, "n_rows: one int32 on the device");
    return (const int32_t*)t.data_ptr();
}
// Codes and scales of `rows` rows of `cols` values.
struct Mx { uint8_t *codes, *scales; int64_t codes_ld, scales_ld; };
Mx mx_of(const Device& dev, const at::Tensor& c, const at::Tensor& s, int64_t rows, int64_t cols) {
    dev.has(c);
    dev.has(s);
    check(c.scalar_type() == at::kByte && s.scalar_type() == at::kByte, "codes, scales: uint8");
    const int64_t cl = row_stride(c, "codes: [rows, cols / 2], rows contiguous"), sl = row_stride(s, "scales: [rows, cols / 32], rows contiguous");
    check(cols % VP_MXFP4_BLOCK == 0, "rows of whole blocks of 32 values are expected");
    check(c.size(0) == rows && s.size(0) == rows && c.size(1) == cols / 2 && s.size(1) == cols / VP_MXFP4_BLOCK,
          "codes: [rows, cols / 2], scales: [rows, cols / 32]");
    return Mx{(uint8_t*)c.data_ptr(), (uint8_t*)s.data_ptr(), cl, sl};
}

// (x, codes, scales, gated, n_rows, stream)
PyObject* mxfp4_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 6, [&] {
        const at::Tensor& x = tensor(a[0]);
        const Device dev(x);
        const int64_t ld = row_stride(x, "x: [rows, cols], rows contiguous");
        const bool gated = integer(a[3]) != 0;
        check(!gated || x.size(1) % 2 == 0, "x: [rows, 2 * cols] when gated");
        const int64_t cols = gated ? x.size(1) / 2 : x.size(1);
        const Mx m = mx_of(dev, tensor(a[1]), tensor(a[2]), x.size(0), cols);
        const int32_t* count = count_of(dev, a[4]);
        const int type = type_of(x);
        void* stream = dev.stream(a[5]);
        int rc;
        WITHOUT_GIL(rc, vp_mxfp4_quantize(x.data_ptr(), type, ld, x.size(0), cols, gated, count, m.codes, m.codes_ld, m.scales, m.scales_ld, stream))
        return rc;
    });
}

// (codes, scales, out, n_rows, stream)
PyObject* mxfp4_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 5, [&] {
        const at::Tensor& out = tensor(a[2]);
        const Device dev(out);
        const int64_t ld = row_stride(out, "out: [rows, cols], rows contiguous");
        const Mx m = mx_of(dev, tensor(a[0]), tensor(a[1]), out.size(0), out.size(1));
        const int32_t* count = count_of(dev, a[3]);
        const int type = type_of(out);
        void* stream = dev.stream(a[4]);
        int rc;
        WITHOUT_GIL(rc, vp_mxfp4_dequantize(m.codes, m.codes_ld, m.scales, m.scales_ld, out.size(0), out.size(1), count, out.data_ptr(), type, ld, stream))
        return rc;
    });
}

// (x_codes, x_scales, w_codes, w_scales, expert_off, out, status, stream)
PyObject* mxfp4_product(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return call(n, 8, [&] {
        const at::Tensor& wc = tensor(a[2]);
        const Device dev(wc);
        const at::Tensor &ws = dev.has(tensor(a[3])), &off = dev.has(tensor(a[4])), &out = dev.has(tensor(a[5])), &st = dev.has(tensor(a[6]));
        check(wc.scalar_type() == at::kByte && wc.is_contiguous() && wc.dim() == 3, "w_codes: contiguous uint8 [E, F, K / 2]");
        const int64_t E = wc.size(0), F = wc.size(1), K = wc.size(2) * 2;
        check(ws.scalar_type() == at::kByte && ws.is_contiguous() && ws.dim() == 3 && ws.size(0) == E && ws.size(1) == F &&
              ws.size(2) == K / VP_MXFP4_BLOCK, "w_scales: contiguous uint8 [E, F, K / 32]");
        const int64_t out_ld = row_stride(out, "out: [capacity_rows, F], rows contiguous");
        check(out.size(1) == F, "out: [capacity_rows, F]");
        const Mx m = mx_of(dev, tensor(a[0]), tensor(a[1]), out.size(0), K);
        check(off.scalar_type() == at::kInt && off.is_contiguous() && off.numel() == E + 1, "expert_off: contiguous int32 [E + 1]");
        check(st.scalar_type() == at::kInt && st.numel() == 1, "status: one int32");
        const int type = type_of(out), e = int_size(E);
        // (a single row needs no stride; the kernel's is a multiple of 16)
        const int64_t codes_ld = out.size(0) <= 1 ? (m.codes_ld + 15) / 16 * 16 : m.codes_ld;
        void* stream = dev.stream(a[7]);
        int rc;
        WITHOUT_GIL(rc, vp_mxfp4_product(m.codes, codes_ld, m.scales, m.scales_ld, out.size(0), (const uint8_t*)wc.data_ptr(),
                                         (const uint8_t*)ws.data_ptr(), e, F, K, (const int32_t*)off.data_ptr(), out.data_ptr(), type, out_ld,
                                         (int32_t*)st.data_ptr(), stream))
        return rc;
    });
}

#define METHOD(n) {#n, (PyCFunction)(void*)n, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(schedule_batch), METHOD(schedule_batch_host), METHOD(schedule_batch_host_used), METHOD(demand_from_routing),
                         METHOD(pack), METHOD(exchange_put), METHOD(unpack), METHOD(unpack_tokens),
                         METHOD(route), METHOD(route_backward), METHOD(combine), METHOD(combine_backward), METHOD(mxfp4_quantize),
                         METHOD(mxfp4_dequantize), METHOD(mxfp4_product), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() {
#define INTERN(n) if (!(s_##n = PyUnicode_InternFromString(#n))) return nullptr;
    NAMES(INTERN)
    return PyModule_Create(&module);
}
