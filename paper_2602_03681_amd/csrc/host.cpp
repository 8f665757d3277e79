// Host path of the calls that are made once per generated token, or per round of drafted tokens: checks, output allocation
// and the call into libnats.so without a trip through Python per argument.
//
// The kernels of a step at small batches take 6 to 8 us; checking fifteen tensors and filling a ctypes call in Python took 12.5
// us per step, which a generation loop then waited for.  The functions here take the arguments of the Python functions
// of the same names by position and return
//   the output tensor   the call was made,
//   an int              it was made and refused: the library's status (its message is in nats_last_error),
//   None                an argument is not what this path takes (a wrong shape, a CPU tensor, a subclass, ...): the Python
//                       function then runs its own checks, which name what is wrong.
// A workspace that the caller did not give is allocated for the call where the step gains by it (see wants_workspace),
// from torch's caching allocator like the output, ordered on the current stream; not while the stream is being captured, where
// torch may have no pool to take it from.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>

#include "nats.h"
#include "nats_serve.h"

namespace {

struct NotTaken {};   // thrown where an argument is not what the fast path takes

const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_CheckExact(o)) throw NotTaken();
    return THPVariable_Unpack(o);
}

void* pointer(const at::Tensor& t, at::ScalarType dt, std::initializer_list<int64_t> shape) {
    if (!t.is_cuda() || t.scalar_type() != dt || t.layout() != at::kStrided ||
        t.sizes() != at::IntArrayRef(shape.begin(), shape.size()) || !t.is_contiguous())
        throw NotTaken();
    return t.data_ptr();
}

void* pointer(PyObject* o, at::ScalarType dt, std::initializer_list<int64_t> shape) { return pointer(tensor(o), dt, shape); }

void* optional(PyObject* o, at::ScalarType dt, std::initializer_list<int64_t> shape) {
    return o == Py_None ? nullptr : pointer(o, dt, shape);
}

double number(PyObject* o) {
    const double x = PyFloat_Check(o) ? PyFloat_AS_DOUBLE(o) : PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) { PyErr_Clear(); throw NotTaken(); }
    return x;
}

int integer(PyObject* o) {
    const long x = PyLong_AsLong(o);
    if ((x == -1 && PyErr_Occurred()) || x != (int)x) { PyErr_Clear(); throw NotTaken(); }
    return (int)x;
}

int dtype_code(at::ScalarType dt) {
    if (dt == at::kFloat) return NATS_F32;
    if (dt == at::kBFloat16) return NATS_BF16;
    throw NotTaken();
}

void* current_stream() { return c10::hip::getCurrentHIPStream().stream(); }

// (an error, as for the null stream beside a capture of another one, counts as capturing)
bool capturing() {
    hipStreamCaptureStatus s = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(c10::hip::getCurrentHIPStream().stream(), &s) == hipSuccess) return s != hipStreamCaptureStatusNone;
    (void)hipGetLastError();
    return true;
}

// Whether a step without a workspace of the caller's gets one: with few (batch, head) pairs one block per pair leaves the
// chip idle.  Measured (bf16, us per step, one block against blocks of 64 rows and a second kernel):
//   d 128, 16 pairs: 64 rows 6.5 / 6.3, 256 rows 8.0 / 6.6, 1000 rows 13.0 / 7.2, 2048 rows 19.6 / 9.0;
//   96 pairs, lengths spread evenly up to the figure: 256 rows 8.7 / 8.2, 1000 rows 14.9 / 10.6, 2048 rows 22.2 / 16.8;
//   192 pairs: 256 rows 10.8 / 11.1 .. 12.6, 1000 rows 19.6 / 17.8 (all equal: 23.4 / 23.5);
//   d 64, 16 pairs: 64 rows 5.1 / 6.1, 256 rows 5.8 / 6.3, 1000 rows 8.5 / 6.7, 2048 rows 12.1 / 7.6.
// The lengths are on the device; what is known here is the capacity.
bool wants_workspace(int64_t pairs, int64_t d, int64_t cap) {
    return d == 128 ? pairs <= 128 && cap >= 128 && cap <= 32768 : pairs <= 64 && cap >= 2048 && cap <= 32768;
}
int64_t small_parts_bytes(int64_t pairs, int64_t d, int64_t cap) {   // one partial result per 64 rows (nats.h)
    return pairs * ((cap + 63) / 64 * (d + 4) + d) * 4;
}

PyObject* status(nats_status st, const at::Tensor& out) {
    if (st != NATS_OK) return PyLong_FromLong(st);
    return THPVariable_Wrap(out);
}

// NotTaken: None; any other C++ exception as torch raises it (an allocation that fails: torch.cuda.OutOfMemoryError)
template <typename F>
PyObject* guarded(F&& f) {
    HANDLE_TH_ERRORS
    try {
        return f();
    } catch (const NotTaken&) {
        Py_RETURN_NONE;
    }
    END_HANDLE_TH_ERRORS
}

// The library's launches without the interpreter lock, as a ctypes call makes them: a launch waits where the stream's queue
// is full, and other threads go on meanwhile.
template <typename F>
nats_status unlocked(F&& f) {
    PyThreadState* const state = PyEval_SaveThread();
    const nats_status st = f();   // (a C entry: throws nothing)
    PyEval_RestoreThread(state);
    return st;
}

// The workspace of a step: the caller's, or one made for the call (kept by the tensor until the call has been enqueued) where
// memory is left for it; the step also runs without.
void set_workspace(nats_dec_params& p, PyObject* given, at::Tensor& own, const at::Tensor& like) {
    if (given != Py_None) {
        const at::Tensor& t = tensor(given);
        if (!t.is_cuda() || t.layout() != at::kStrided || !t.is_contiguous()) throw NotTaken();
        p.workspace = t.data_ptr();
        p.workspace_bytes = (size_t)t.numel();
    } else if (wants_workspace((int64_t)p.B * p.H, p.d, p.cap) && !capturing()) {
        const int64_t bytes = small_parts_bytes((int64_t)p.B * p.H, p.d, p.cap);
        try {
            own = at::empty({bytes}, like.options().dtype(at::kByte));
        } catch (const c10::OutOfMemoryError&) {
            return;
        }
        p.workspace = own.data_ptr();
        p.workspace_bytes = (size_t)bytes;
    }
}

void set_scalars(nats_dec_params& p, PyObject* const* a) {   // softmax_scale, la_scale, combine_mode, rms_eps, linear_op
    p.softmax_scale = (float)number(a[0]);
    p.la_scale = (float)number(a[1]);
    p.combine_mode = integer(a[2]);
    p.rms_eps = (float)number(a[3]);
    p.linear_op = integer(a[4]);
}

// decode(state, k_cache, v_cache, cache_len, q, k, v, alpha, beta, mask, q_nla, k_nla, w_nla, w_la, out, err_flags,
//        workspace, softmax_scale, la_scale, combine_mode, rms_eps, linear_op, freeze_on_softmax)
PyObject* decode(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 23) throw NotTaken();
        const at::Tensor& kc = tensor(a[1]);
        if (kc.dim() != 4) throw NotTaken();
        const int64_t B = kc.size(0), H = kc.size(1), cap = kc.size(2), d = kc.size(3);
        const at::ScalarType dt = kc.scalar_type();
        nats_dec_params p{};
        p.B = (int)B; p.H = (int)H; p.d = (int)d; p.cap = (int)cap; p.dtype = dtype_code(dt);
        void* state = pointer(a[0], at::kFloat, {B, H, d, d});
        void* kcache = pointer(kc, dt, {B, H, cap, d});
        void* vcache = pointer(a[2], dt, {B, H, cap, d});
        void* len = pointer(a[3], at::kInt, {B, H});
        const at::Tensor& q = tensor(a[4]);
        void* qp = pointer(q, dt, {B, H, d});
        void* kp = pointer(a[5], dt, {B, H, d});
        void* vp = pointer(a[6], dt, {B, H, d});
        void* alpha = pointer(a[7], at::kFloat, {B, H});
        void* beta = pointer(a[8], at::kFloat, {B, H});
        void* mask = pointer(a[9], at::kByte, {B, H});
        p.q_nla = optional(a[10], dt, {B, H, d});
        p.k_nla = optional(a[11], dt, {B, H, d});
        void* wn = optional(a[12], at::kFloat, {B, H});
        void* wl = optional(a[13], at::kFloat, {B, H});
        void* err = optional(a[15], at::kInt, {B, H});
        set_scalars(p, a + 17);
        p.freeze_on_softmax = integer(a[22]);
        const at::Tensor out = a[14] == Py_None ? at::empty({B, H, d}, q.options()) : tensor(a[14]);
        void* op = pointer(out, dt, {B, H, d});
        at::Tensor own;
        set_workspace(p, a[16], own, q);
        void* const stream = current_stream();
        return status(unlocked([&] {
            return nats_hybrid_attn_decode(&p, (float*)state, kcache, vcache, (int32_t*)len, qp, kp, vp, (const float*)alpha,
                                           (const float*)beta, (const uint8_t*)mask, (const float*)wn, (const float*)wl, op,
                                           (int32_t*)err, stream);
        }), out);
    });
}

PyObject* item(PyObject* dict, const char* key) {
    PyObject* o = PyDict_GetItemString(dict, key);   // borrowed
    if (o == nullptr) throw NotTaken();
    return o;
}

// decode_chunk(st, q, k, v, alpha, beta, w_nla, w_la, out, err_flags, softmax_scale, la_scale, combine_mode, rms_eps, linear_op)
PyObject* decode_chunk(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 15 || !PyDict_CheckExact(a[0])) throw NotTaken();
        const at::Tensor& kc = tensor(item(a[0], "k_cache"));
        if (kc.dim() != 4) throw NotTaken();
        const int64_t B = kc.size(0), H = kc.size(1), cap = kc.size(2), d = kc.size(3);
        const at::ScalarType dt = kc.scalar_type();
        nats_dec_params p{};
        p.B = (int)B; p.H = (int)H; p.d = (int)d; p.cap = (int)cap; p.dtype = dtype_code(dt);
        nats_dec_chunk_state s{};
        s.state = (float*)pointer(item(a[0], "state"), at::kFloat, {B, H, d, d});
        s.state_start = (float*)pointer(item(a[0], "state_start"), at::kFloat, {B, H, d, d});
        s.chunk_decay = (float*)pointer(item(a[0], "chunk_decay"), at::kFloat, {B, H});
        s.chunk_pos = (int32_t*)pointer(item(a[0], "chunk_pos"), at::kInt, {B, H});
        s.k_cache = pointer(kc, dt, {B, H, cap, d});
        s.v_cache = pointer(item(a[0], "v_cache"), dt, {B, H, cap, d});
        s.cache_len = (int32_t*)pointer(item(a[0], "cache_len"), at::kInt, {B, H});
        const at::Tensor& q = tensor(a[1]);
        void* qp = pointer(q, dt, {B, H, d});
        void* kp = pointer(a[2], dt, {B, H, d});
        void* vp = pointer(a[3], dt, {B, H, d});
        void* alpha = pointer(a[4], at::kFloat, {B, H});
        void* beta = pointer(a[5], at::kFloat, {B, H});
        void* wn = optional(a[6], at::kFloat, {B, H});
        void* wl = optional(a[7], at::kFloat, {B, H});
        void* err = optional(a[9], at::kInt, {B, H});
        set_scalars(p, a + 10);
        const at::Tensor out = a[8] == Py_None ? at::empty({B, H, d}, q.options()) : tensor(a[8]);
        void* op = pointer(out, dt, {B, H, d});
        at::Tensor own;
        set_workspace(p, Py_None, own, q);
        void* const stream = current_stream();
        return status(unlocked([&] {
            return nats_hybrid_attn_decode_chunk(&p, &s, qp, kp, vp, (const float*)alpha, (const float*)beta, (const float*)wn,
                                                 (const float*)wl, op, (int32_t*)err, stream);
        }), out);
    });
}

// ---- the calls of nats_serve.h: tensors on the current device only ----
struct Here {
    c10::DeviceIndex device = -1;   // asked for behind the first tensor that is on a GPU: without one there is no device to ask for
    void* operator()(const at::Tensor& t, at::ScalarType dt, std::initializer_list<int64_t> shape) {
        void* const p = pointer(t, dt, shape);
        if (device < 0) device = c10::hip::current_device();
        if (t.device().index() != device) throw NotTaken();
        return p;
    }
    void* operator()(PyObject* o, at::ScalarType dt, std::initializer_list<int64_t> shape) { return (*this)(tensor(o), dt, shape); }
    void* optional(PyObject* o, at::ScalarType dt, std::initializer_list<int64_t> shape) {
        return o == Py_None ? nullptr : (*this)(o, dt, shape);
    }
    // the caller's workspace, or one made for the call
    void* workspace(PyObject* given, at::Tensor& own, const at::Tensor& like, size_t need, size_t& bytes) {
        if (given == Py_None) {
            bytes = need;
            if (need == 0) return nullptr;
            own = at::empty({(int64_t)need}, like.options().dtype(at::kByte));
            return own.data_ptr();
        }
        const at::Tensor& t = tensor(given);
        if (!t.is_cuda() || t.layout() != at::kStrided || !t.is_contiguous() || t.device().index() != device) throw NotTaken();
        bytes = (size_t)t.numel();
        return t.data_ptr();
    }
};

at::Tensor given_or_new(PyObject* o, std::initializer_list<int64_t> shape, const at::Tensor& like, at::ScalarType dt) {
    return o == Py_None ? at::empty(at::IntArrayRef(shape.begin(), shape.size()), like.options().dtype(dt)) : tensor(o);
}

// B, H, T, d, cap, dtype, group of a call on a tree (k [B,H,T,d], k_cache [B,H group,cap,d])
void tree_sizes(nats_tree_params& p, const at::Tensor& k, const at::Tensor& kc, int group) {
    if (kc.dim() != 4 || k.dim() != 4 || group < 1 || k.size(1) * group != kc.size(1)) throw NotTaken();
    p.B = (int)kc.size(0); p.H = (int)k.size(1); p.T = (int)k.size(2); p.d = (int)kc.size(3); p.cap = (int)kc.size(2);
    p.dtype = dtype_code(kc.scalar_type());
    p.group = group;
}

// decode_tree(state, k_cache, v_cache, cache_len, q, k, v, alpha, beta, mask, parent, n_nodes, q_nla, k_nla, w_nla, w_la, out, lse,
//             workspace, softmax_scale, la_scale, combine_mode, rms_eps, linear_op, freeze_on_softmax, group) -> (out, lse)
PyObject* decode_tree(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 26) throw NotTaken();
        Here here;
        const at::Tensor &kc = tensor(a[1]), &k = tensor(a[5]), &v = tensor(a[6]);
        nats_tree_params p{};
        tree_sizes(p, k, kc, integer(a[25]));
        const int64_t B = p.B, H = p.H, T = p.T, d = p.d, cap = p.cap, HG = kc.size(1);
        const at::ScalarType dt = kc.scalar_type();
        void* state = here(a[0], at::kFloat, {B, HG, d, d});
        void* kcache = here(kc, dt, {B, HG, cap, d});
        void* vcache = here(a[2], dt, {B, HG, cap, d});
        void* len = here(a[3], at::kInt, {B, HG});
        void* qp = here(a[4], dt, {B, H, T, d});
        void* kp = here(k, dt, {B, H, T, d});
        void* vp = here(v, dt, {B, HG, T, d});
        void* alpha = here(a[7], at::kFloat, {B, H, T});
        void* beta = here(a[8], at::kFloat, {B, H, T});
        void* mask = here(a[9], at::kByte, {B, H, T});
        void* parent = here(a[10], at::kInt, {B, T});
        void* nodes = here.optional(a[11], at::kInt, {B});
        p.q_nla = here.optional(a[12], dt, {B, HG, T, d});
        p.k_nla = here.optional(a[13], dt, {B, HG, T, d});
        void* wn = here.optional(a[14], at::kFloat, {B, HG, T});
        void* wl = here.optional(a[15], at::kFloat, {B, HG, T});
        p.softmax_scale = (float)number(a[19]);
        p.la_scale = (float)number(a[20]);
        p.combine_mode = integer(a[21]);
        p.rms_eps = (float)number(a[22]);
        p.linear_op = integer(a[23]);
        p.freeze_on_softmax = integer(a[24]);
        const at::Tensor out = given_or_new(a[16], {B, HG, T, d}, v, dt), lse = given_or_new(a[17], {B, HG, T}, v, at::kFloat);
        void* op = here(out, dt, {B, HG, T, d});
        void* lp = here(lse, at::kFloat, {B, HG, T});
        at::Tensor own;
        size_t bytes = 0;
        const size_t need = a[18] == Py_None ? nats_hybrid_attn_decode_tree_workspace_bytes(&p) : 0;
        void* const ws = here.workspace(a[18], own, v, need, bytes);
        void* const stream = current_stream();
        const nats_status st = unlocked([&] {
            return nats_hybrid_attn_decode_tree(&p, (const float*)state, kcache, vcache, (const int32_t*)len, qp, kp, vp, (const float*)alpha,
                                                (const float*)beta, (const uint8_t*)mask, (const int32_t*)parent, (const int32_t*)nodes,
                                                (const float*)wn, (const float*)wl, op, (float*)lp, ws, bytes, stream);
        });
        if (st != NATS_OK) return PyLong_FromLong(st);
        PyObject* pair[2] = {THPVariable_Wrap(out), THPVariable_Wrap(lse)};
        PyObject* const r = pair[0] && pair[1] ? PyTuple_Pack(2, pair[0], pair[1]) : nullptr;
        Py_XDECREF(pair[0]);
        Py_XDECREF(pair[1]);
        return r;
    });
}

// tree_commit(state, k_cache, v_cache, cache_len, k, v, alpha, beta, mask, parent, node, n_nodes, k_nla, vis, err_flags, linear_op,
//             freeze_on_softmax, group) -> vis
PyObject* tree_commit(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 18) throw NotTaken();
        Here here;
        const at::Tensor &kc = tensor(a[1]), &k = tensor(a[4]), &v = tensor(a[5]);
        nats_tree_params p{};
        tree_sizes(p, k, kc, integer(a[17]));
        const int64_t B = p.B, H = p.H, T = p.T, d = p.d, cap = p.cap, HG = kc.size(1);
        const at::ScalarType dt = kc.scalar_type();
        void* state = here(a[0], at::kFloat, {B, HG, d, d});
        void* kcache = here(kc, dt, {B, HG, cap, d});
        void* vcache = here(a[2], dt, {B, HG, cap, d});
        void* len = here(a[3], at::kInt, {B, HG});
        void* kp = here(k, dt, {B, H, T, d});
        void* vp = here(v, dt, {B, HG, T, d});
        void* alpha = here(a[6], at::kFloat, {B, H, T});
        void* beta = here(a[7], at::kFloat, {B, H, T});
        void* mask = here(a[8], at::kByte, {B, H, T});
        void* parent = here(a[9], at::kInt, {B, T});
        void* node = here(a[10], at::kInt, {B});
        void* nodes = here.optional(a[11], at::kInt, {B});
        p.k_nla = here.optional(a[12], dt, {B, HG, T, d});
        void* err = here.optional(a[14], at::kInt, {B, HG});
        p.linear_op = integer(a[15]);
        p.freeze_on_softmax = integer(a[16]);
        const at::Tensor vis = given_or_new(a[13], {B, HG, T}, v, at::kInt);
        void* visp = here(vis, at::kInt, {B, HG, T});
        void* const stream = current_stream();
        return status(unlocked([&] {
            return nats_hybrid_attn_tree_commit_ex(&p, (float*)state, kcache, vcache, (int32_t*)len, kp, vp, (const float*)alpha,
                                                   (const float*)beta, (const uint8_t*)mask, (const int32_t*)parent,
                                                   (const int32_t*)nodes, (const int32_t*)node, (int32_t*)visp, (int32_t*)err, stream);
        }), vis);
    });
}

// cache_weights(weights, q, k_cache, cache_len, lse, vis, workspace, softmax_scale, decay) -> weights
PyObject* cache_weights(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 9) throw NotTaken();
        Here here;
        const at::Tensor &weights = tensor(a[0]), &q = tensor(a[1]), &kc = tensor(a[2]);
        if (kc.dim() != 4 || q.dim() != 4) throw NotTaken();
        const int64_t B = kc.size(0), H = kc.size(1), cap = kc.size(2), d = kc.size(3), Hq = q.size(1), T = q.size(2);
        int64_t Hv = H;
        if (a[5] != Py_None) {
            if (tensor(a[5]).dim() != 3) throw NotTaken();
            Hv = tensor(a[5]).size(1);
        }
        if (Hq == 0 || Hv == 0 || H % Hq || H % Hv) throw NotTaken();
        const at::ScalarType dt = kc.scalar_type();
        nats_cache_weights_params p{};
        p.B = (int)B; p.H = (int)H; p.T = (int)T; p.d = (int)d; p.cap = (int)cap; p.dtype = dtype_code(dt);
        p.q_group = (int)(H / Hq);
        p.vis_group = (int)(H / Hv);
        p.softmax_scale = (float)number(a[7]);
        p.decay = (float)number(a[8]);
        void* wp = here(weights, at::kFloat, {B, H, cap});
        void* qp = here(q, dt, {B, Hq, T, d});
        void* kp = here(kc, dt, {B, H, cap, d});
        void* len = here(a[3], at::kInt, {B, H});
        void* lse = here.optional(a[4], at::kFloat, {B, H, T});
        void* vis = here.optional(a[5], at::kInt, {B, Hv, T});
        at::Tensor own;
        size_t bytes = 0;
        const size_t need = a[6] == Py_None ? nats_cache_weights_workspace_bytes(&p, lse != nullptr) : 0;
        void* const ws = here.workspace(a[6], own, q, need, bytes);
        void* const stream = current_stream();
        return status(unlocked([&] {
            return nats_cache_weights(&p, (float*)wp, qp, kp, (const int32_t*)len, (const int32_t*)vis, (const float*)lse, ws, bytes, stream);
        }), weights);
    });
}

// cache_evict(k_cache, v_cache, cache_len, weights, kept, keep, recent, clear_weights) -> kept
PyObject* cache_evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        if (n != 8) throw NotTaken();
        Here here;
        const at::Tensor& kc = tensor(a[0]);
        if (kc.dim() != 4) throw NotTaken();
        const int64_t B = kc.size(0), H = kc.size(1), cap = kc.size(2), d = kc.size(3);
        const at::ScalarType dt = kc.scalar_type();
        nats_cache_evict_params p{(int)B, (int)H, (int)d, (int)cap, dtype_code(dt), integer(a[5]), integer(a[6])};
        if (p.keep < 1 || p.keep > cap) throw NotTaken();
        void* kp = here(kc, dt, {B, H, cap, d});
        void* vp = here(a[1], dt, {B, H, cap, d});
        void* len = here(a[2], at::kInt, {B, H});
        void* wp = here(a[3], at::kFloat, {B, H, cap});
        const at::Tensor kept = given_or_new(a[4], {B, H, (int64_t)p.keep}, kc, at::kInt);
        void* keptp = here(kept, at::kInt, {B, H, (int64_t)p.keep});
        const auto evict = integer(a[7]) ? nats_cache_evict_clear : nats_cache_evict;
        void* const stream = current_stream();
        return status(unlocked([&] { return evict(&p, kp, vp, (int32_t*)len, (float*)wp, (int32_t*)keptp, stream); }), kept);
    });
}

PyMethodDef methods[] = {
    {"decode", (PyCFunction)(void (*)(void))decode, METH_FASTCALL, "nats_hybrid_attn_decode"},
    {"decode_chunk", (PyCFunction)(void (*)(void))decode_chunk, METH_FASTCALL, "nats_hybrid_attn_decode_chunk"},
    {"decode_tree", (PyCFunction)(void (*)(void))decode_tree, METH_FASTCALL, "nats_hybrid_attn_decode_tree"},
    {"tree_commit", (PyCFunction)(void (*)(void))tree_commit, METH_FASTCALL, "nats_hybrid_attn_tree_commit"},
    {"cache_weights", (PyCFunction)(void (*)(void))cache_weights, METH_FASTCALL, "nats_cache_weights"},
    {"cache_evict", (PyCFunction)(void (*)(void))cache_evict, METH_FASTCALL, "nats_cache_evict"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_nats_host", "host path of the per-token calls", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__nats_host() { return PyModule_Create(&module); }
