// The argument marshalling of binding.py's calls in native code: checks, fresh outputs and the C call of one entry point per
// function, for the ordinary form of a call.  What is not of that form -- another tensor type or place, a shape or an output
// that does not fit, numbers that are not Python numbers -- is declined (None) before anything has happened, and binding.py
// goes through it step by step, with its own checks and messages.  A call that the library refuses returns its code.
// Everything that can fail, the Python objects of the results included, is done before the library is called: a failure behind
// the launch, taken for a declined call, would have binding.py launch it a second time.
//
// Why: of the 26 us of the smallest stage-1 call 18 were Python (eleven outputs and a workspace of 1.2 us each, 31 ctypes
// arguments), of one pruning level's 28 us of host time 15; the kernels of both take less than that.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "metok.h"
#include "metok_decode.h"
#include "metok_qkv.h"

namespace {

// Thrown and caught inside this file only.  A Python error is never a reason to decline: it may be a signal's exception.
struct Declined {};
struct Raised {};                          // a Python error is set

// ---- reading arguments -----------------------------------------------------------------------------------------------
inline void need(bool ok) { if (!ok) throw Declined(); }

inline int64_t integer(PyObject* o) {
    need(PyLong_CheckExact(o) || PyBool_Check(o));
    int overflow = 0;
    const int64_t v = PyLong_AsLongLongAndOverflow(o, &overflow);
    need(!overflow);
    return v;
}
inline int int32(PyObject* o) {
    const int64_t v = integer(o);
    need(v >= INT32_MIN && v <= INT32_MAX);
    return static_cast<int>(v);
}
inline double real(PyObject* o) {
    if (PyFloat_CheckExact(o)) return PyFloat_AS_DOUBLE(o);
    return static_cast<double>(int32(o));
}
inline bool given(PyObject* o) { return o != Py_None; }

struct Owned {                             // a reference of our own, to what a Python function returned
    PyObject* o;
    explicit Owned(PyObject* p) : o(p) { if (!o) throw Raised(); }
    Owned(const Owned&) = delete;
    ~Owned() { Py_XDECREF(o); }
    PyObject* release() { PyObject* p = o; o = nullptr; return p; }
};

// A plain tensor on the GPU, contiguous.
inline const at::Tensor& tensor(PyObject* o) {
    need(THPVariable_CheckExact(o));
    const at::Tensor& t = THPVariable_Unpack(o);
    need(t.is_cuda() && t.layout() == at::kStrided && t.is_contiguous());
    return t;
}
inline void* address(const at::Tensor& t) { return t.data_ptr(); }
inline int dtype_code(const at::Tensor& t) {
    const auto s = t.scalar_type();
    need(s == at::kBFloat16 || s == at::kFloat);
    return s == at::kBFloat16 ? METOK_BF16 : METOK_F32;
}

// The caller's outputs: None, or a dict.
struct Outputs {
    PyObject* dict;                        // borrowed, nullptr: none given
    at::Device device;
    Outputs(PyObject* o, const at::Tensor& like) : dict(given(o) ? o : nullptr), device(like.device()) { need(!dict || PyDict_CheckExact(dict)); }
    PyObject* find(const char* name) const {
        if (!dict) return nullptr;
        const Owned key(PyUnicode_FromString(name));
        PyObject* v = PyDict_GetItemWithError(dict, key.o);  // borrowed
        if (!v && PyErr_Occurred()) throw Raised();
        return v && given(v) ? v : nullptr;
    }
    at::Tensor fresh(at::IntArrayRef shape, at::ScalarType type) const {
        for (const int64_t n : shape) need(n >= 0);
        return at::empty(shape, at::TensorOptions().dtype(type).device(device));
    }
    at::Tensor get(const char* name, at::IntArrayRef shape, at::ScalarType type) const {
        if (PyObject* v = find(name)) {
            const at::Tensor& t = tensor(v);
            need(t.scalar_type() == type && t.sizes() == shape);
            return t;
        }
        return fresh(shape, type);
    }
};
inline at::Tensor workspace_of(PyObject* o, const Outputs& out, size_t bytes) {
    if (given(o)) return tensor(o);
    return out.fresh({static_cast<int64_t>(std::max<size_t>(bytes, 256))}, at::kByte);
}

// ---- results -----------------------------------------------------------------------------------------------------------
struct Result : Owned {
    Result() : Owned(PyDict_New()) {}
    void put(const char* name, PyObject* v) {                // takes the reference
        const Owned own(v);
        if (PyDict_SetItemString(o, name, v)) throw Raised();
    }
    void put(const char* name, const at::Tensor& t) { put(name, THPVariable_Wrap(t)); }
};

// A call with its arguments, pointers among them, read now.
template <typename F, typename... A> auto bound(F f, A... a) { return [=] { return f(a...); }; }

// The library call of one native call, without the interpreter's lock, as ctypes does.
struct Launch {
    bool made = false;
    template <typename F> int operator()(F&& call) {
        struct Released {
            PyThreadState* state = PyEval_SaveThread();
            ~Released() { PyEval_RestoreThread(state); }
        } released;
        made = true;
        return call();
    }
};
// The library's code, unless it is 0: then the results.
inline PyObject* answer(int rc, Owned& results) { return rc ? PyLong_FromLong(rc) : results.release(); }

template <typename F> PyObject* guarded(Py_ssize_t nargs, Py_ssize_t expected, F&& body) {
    if (nargs != expected) { PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", expected, nargs); return nullptr; }
    Launch launch;
    try {
        return body(launch);
    } catch (const Raised&) {
        return nullptr;
    } catch (python_error& e) {            // torch's form of the same
        e.restore();
        return nullptr;
    } catch (const Declined&) {
        Py_RETURN_NONE;
    } catch (const std::exception& e) {    // an allocation that failed, for instance: the step-by-step path reports it
        if (launch.made) { PyErr_SetString(PyExc_RuntimeError, e.what()); return nullptr; }      // not again
        Py_RETURN_NONE;
    }
}
// binding.py's function for the current stream's handle, asked once everything else fits.
inline void* stream_of(PyObject* f) {
    const Owned handle(PyObject_CallNoArgs(f));
    return reinterpret_cast<void*>(integer(handle.o));
}

// binding.py's function for the stream of a device that has to be the current one, None if it is not: binding.py says so then.
inline void* stream_on(PyObject* f, const at::Tensor& t) {
    const Owned index(PyLong_FromLong(t.device().index()));
    const Owned handle(PyObject_CallOneArg(f, index.o));
    return reinterpret_cast<void*>(integer(handle.o));
}

// ---- stage 1 -----------------------------------------------------------------------------------------------------------
// feats, grid_h, grid_w, k, text_emb, alpha, beta, s1, s2, sim_mode, event_reduce, pool_edge, workspace, out, stream
template <bool BATCHED>
PyObject* segment_compress(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 15, [&](Launch& launch) -> PyObject* {
        const at::Tensor& feats = tensor(a[0]);
        const at::Tensor& text = tensor(a[4]);
        need(feats.dim() == (BATCHED ? 4 : 3));
        const int64_t B = BATCHED ? feats.size(0) : 1, T = feats.size(BATCHED), N = feats.size(BATCHED + 1), d = feats.size(BATCHED + 2);
        const int64_t limit = INT32_MAX;
        need(B <= limit && T <= limit && N <= limit && d <= limit);
        const int gh = int32(a[1]), gw = int32(a[2]), k = int32(a[3]), s1 = int32(a[7]), s2 = int32(a[8]);
        const double alpha = real(a[5]), beta = real(a[6]);
        const int sim_mode = int32(a[9]), reduce = int32(a[10]), edge = int32(a[11]), dt = dtype_code(feats);
        need(static_cast<int64_t>(gh) * gw == N);
        if (BATCHED) need(text.dim() == 2 && text.size(0) == B && text.size(1) == d);
        const int64_t cap = metok_compress_encoder_tokens_capacity_rows(static_cast<int>(T), gh, gw, s1, s2, edge);
        need(cap >= 0 && k >= 0);
        const Outputs out(a[13], feats);
        at::Tensor tokens;
        if (PyObject* v = out.find("out_tokens")) {
            tokens = tensor(v);
            need(tokens.dim() == (BATCHED ? 3 : 2) && tokens.size(BATCHED + 1) == d && (!BATCHED || tokens.size(0) == B));
        } else {
            tokens = BATCHED ? out.fresh({B, cap, d}, feats.scalar_type()) : out.fresh({cap, d}, feats.scalar_type());
        }
        const int odt = dtype_code(tokens);
        const int64_t rows = tokens.size(BATCHED);
        const at::Tensor ws = workspace_of(a[12], out, BATCHED ? metok_segment_compress_batched_workspace_bytes(static_cast<int>(B), static_cast<int>(T), gh, gw, static_cast<int>(d), dt)
                                                               : metok_segment_compress_workspace_bytes(static_cast<int>(T), gh, gw, static_cast<int>(d), dt));
        auto get = [&](const char* name, int64_t len, at::ScalarType type) {
            const int64_t shape[2] = {B, len};
            return out.get(name, BATCHED ? at::IntArrayRef(shape, 2) : at::IntArrayRef(shape + 1, 1), type);
        };
        const at::Tensor token_event = get("token_event", rows, at::kInt), frame_event = get("frame_event", T, at::kInt), frame_stride = get("frame_stride", T, at::kInt),
                         event_start = get("event_start", k + 1, at::kInt), frame_offsets = get("frame_offsets", T + 1, at::kInt),
                         frame_is_key = get("frame_is_key", T, at::kByte), event_is_key = get("event_is_key", k, at::kByte),
                         frame_score = get("frame_score", T, at::kFloat), sim = get("sim", std::max<int64_t>(T - 1, 0), at::kFloat),
                         event_score = get("event_score", k, at::kFloat);
        Result r;
        r.put("sim", sim); r.put("event_start", event_start); r.put("frame_event", frame_event); r.put("out_tokens", tokens);
        r.put("frame_offsets", frame_offsets); r.put("token_event", token_event); r.put("event_is_key", event_is_key); r.put("frame_is_key", frame_is_key);
        r.put("frame_stride", frame_stride); r.put("event_score", event_score); r.put("frame_score", frame_score);
        void* stream = stream_of(a[14]);
        auto call = [&](auto... first) {
            return bound(first..., address(feats), dt, static_cast<int>(T), gh, gw, static_cast<int>(d), address(text), k, sim_mode, alpha, beta, s1, s2, reduce, edge,
                         static_cast<float*>(address(sim)), static_cast<int32_t*>(address(event_start)), static_cast<int32_t*>(address(frame_event)), address(tokens), rows, odt,
                         static_cast<int32_t*>(address(frame_offsets)), static_cast<int32_t*>(address(token_event)), static_cast<uint8_t*>(address(event_is_key)),
                         static_cast<uint8_t*>(address(frame_is_key)), static_cast<int32_t*>(address(frame_stride)), static_cast<float*>(address(event_score)),
                         static_cast<float*>(address(frame_score)), address(ws), static_cast<size_t>(ws.numel()), stream);
        };
        int rc;
        if constexpr (BATCHED) rc = launch(call(&metok_segment_compress_batched, static_cast<int>(B)));
        else rc = launch(call(&metok_segment_compress));
        return answer(rc, r);
    });
}

// ---- stage 2 -----------------------------------------------------------------------------------------------------------
// The quotas of one video, appended; returns their sum.
int64_t quotas_of(PyObject* o, std::vector<int32_t>& all) {
    need(PyList_CheckExact(o) || PyTuple_CheckExact(o));
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(o);
    PyObject** items = PySequence_Fast_ITEMS(o);
    int64_t total = 0;
    for (Py_ssize_t i = 0; i < n; ++i) { const int q = int32(items[i]); all.push_back(q); total += q; }
    return total;
}

// hidden, vis_start, n_vis, token_seg, seg_quota, q_text, k_all, token_event, event_weight, orig_idx, scores, hidden_out, workspace, out,
// score_mode, static_scratch, stream
PyObject* prefill_prune(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 17, [&](Launch& launch) -> PyObject* {
        const at::Tensor& hidden = tensor(a[0]);
        const at::Tensor& seg = tensor(a[3]);
        need(hidden.dim() == 2);
        const int64_t S = hidden.size(0), D = hidden.size(1);
        need(D <= INT32_MAX);
        const int vis_start = int32(a[1]), n_vis = int32(a[2]), mode = int32(a[14]), dt = dtype_code(hidden);
        const bool fixed = integer(a[15]) != 0;
        std::vector<int32_t> quota;
        const int64_t total = quotas_of(a[4], quota);
        const Outputs out(a[13], hidden);
        at::Tensor q, keys, scores, event, weight, orig;
        int Hq = 0, Hkv = 0, dh = 0, Tq = 0;
        if (given(a[5])) {
            q = tensor(a[5]); keys = tensor(a[6]);
            need(q.dim() == 3 && keys.dim() == 3 && keys.size(1) == S && keys.size(2) == q.size(2) && dtype_code(q) == dt && dtype_code(keys) == dt);
            for (int i = 0; i < 3; ++i) need(q.size(i) <= INT32_MAX && keys.size(i) <= INT32_MAX);
            Hq = static_cast<int>(q.size(0)); Tq = static_cast<int>(q.size(1)); dh = static_cast<int>(q.size(2)); Hkv = static_cast<int>(keys.size(0));
            scores = out.get("scores", {n_vis}, at::kFloat);
        } else {
            need(!given(a[6]));
            scores = tensor(a[10]);
        }
        if (given(a[7])) event = tensor(a[7]);
        if (given(a[8])) weight = tensor(a[8]);
        if (given(a[9])) orig = tensor(a[9]);
        at::Tensor ws;
        if (!fixed) ws = workspace_of(a[12], out, given(a[12]) ? 0 : metok_prefill_prune_workspace_bytes(S, Hq, Hkv, dh, Tq, n_vis, dt));
        const at::Tensor kept = out.get("kept_idx", {total}, at::kInt), seg_out = out.get("token_seg_out", {total}, at::kInt), orig_out = out.get("orig_idx_out", {total}, at::kInt);
        at::Tensor event_out;
        if (event.defined()) event_out = out.get("token_event_out", {total}, at::kInt);
        const int64_t rows = S - n_vis + total;
        at::Tensor hidden_out;
        PyObject* ho = given(a[11]) ? a[11] : out.find("hidden_out");
        if (ho) {
            hidden_out = tensor(ho);
            need(hidden_out.dim() == 2 && hidden_out.size(0) == rows && hidden_out.size(1) == D && hidden_out.scalar_type() == hidden.scalar_type());
        } else {
            hidden_out = out.fresh({rows, D}, hidden.scalar_type());
        }
        auto at_ = [](const at::Tensor& t) -> void* { return t.defined() ? address(t) : nullptr; };
        const int n_events = weight.defined() ? static_cast<int>(weight.numel()) : 0;
        Result r;
        r.put("scores", scores); r.put("kept_idx", kept);
        if (ho) { Py_INCREF(ho); r.put("hidden_out", ho); } else r.put("hidden_out", hidden_out);
        r.put("token_seg_out", seg_out); r.put("orig_idx_out", orig_out);
        if (event_out.defined()) r.put("token_event_out", event_out);
        void* stream = stream_of(a[16]);
        auto call = [&](auto f, auto... last) {
            return bound(f, address(hidden), S, static_cast<int>(D), dt, at_(q), at_(keys), Hq, Hkv, dh, Tq, mode, vis_start, n_vis, static_cast<const int32_t*>(address(seg)),
                         static_cast<const int32_t*>(at_(event)), static_cast<const float*>(at_(weight)), n_events, static_cast<int>(quota.size()), quota.data(),
                         static_cast<const int32_t*>(at_(orig)), static_cast<float*>(address(scores)), static_cast<int32_t*>(address(kept)), address(hidden_out),
                         static_cast<int32_t*>(address(seg_out)), static_cast<int32_t*>(at_(event_out)), static_cast<int32_t*>(address(orig_out)), last...);
        };
        return answer(fixed ? launch(call(&metok_prefill_prune_static, stream))
                            : launch(call(&metok_prefill_prune, address(ws), static_cast<size_t>(ws.numel()), stream)), r);
    });
}

// hidden, vis_start, n_vis, token_seg, seg_quota, q_text, k_all, token_event, event_weight, orig_idx, scores, hidden_out, workspace, out,
// score_mode, keep_stride, out_row_stride, stream
PyObject* prefill_prune_batched(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 18, [&](Launch& launch) -> PyObject* {
        const at::Tensor& hidden = tensor(a[0]);
        const at::Tensor& seg = tensor(a[3]);
        need(hidden.dim() == 3);
        const int64_t B = hidden.size(0), S = hidden.size(1), D = hidden.size(2);
        need(B >= 1 && B <= METOK_MAX_BATCH && D <= INT32_MAX);
        const int vis_start = int32(a[1]), n_vis = int32(a[2]), mode = int32(a[14]), dt = dtype_code(hidden);
        need(PyList_CheckExact(a[4]) || PyTuple_CheckExact(a[4]));
        need(PySequence_Fast_GET_SIZE(a[4]) == B);
        std::vector<int32_t> quota;
        std::vector<int64_t> keep;
        int64_t most = 0;
        for (int64_t b = 0; b < B; ++b) {
            keep.push_back(quotas_of(PySequence_Fast_ITEMS(a[4])[b], quota));
            most = b ? std::max(most, keep[b]) : keep[0];
        }
        const int n_seg = static_cast<int>(quota.size() / B);
        for (int64_t b = 0; b < B; ++b) need(PySequence_Fast_GET_SIZE(PySequence_Fast_ITEMS(a[4])[b]) == n_seg);
        const Outputs out(a[13], hidden);
        auto is = [](const at::Tensor& t, int64_t r, int64_t c) { return t.dim() == 2 && t.size(0) == r && t.size(1) == c; };
        at::Tensor q, keys, scores, event, weight, orig;
        int Hq = 0, Hkv = 0, dh = 0, Tq = 0;
        if (given(a[5])) {
            q = tensor(a[5]); keys = tensor(a[6]);
            need(q.dim() == 4 && keys.dim() == 4 && q.size(0) == B && keys.size(0) == B && keys.size(2) == S && keys.size(3) == q.size(3) && dtype_code(q) == dt && dtype_code(keys) == dt);
            for (int i = 0; i < 4; ++i) need(q.size(i) <= INT32_MAX && keys.size(i) <= INT32_MAX);
            Hq = static_cast<int>(q.size(1)); Tq = static_cast<int>(q.size(2)); dh = static_cast<int>(q.size(3)); Hkv = static_cast<int>(keys.size(1));
            scores = out.get("scores", {B, n_vis}, at::kFloat);
        } else {
            need(!given(a[6]));
            scores = tensor(a[10]);
            need(is(scores, B, n_vis));
        }
        need(is(seg, B, n_vis));
        if (given(a[7])) { event = tensor(a[7]); need(is(event, B, n_vis)); }
        if (given(a[8])) { weight = tensor(a[8]); need(weight.dim() == 2 && weight.size(0) == B && weight.size(1) <= INT32_MAX); }
        if (given(a[9])) { orig = tensor(a[9]); need(orig.dim() == 2 && orig.size(0) == B && orig.size(1) >= n_vis); }
        const at::Tensor ws = workspace_of(a[12], out, given(a[12]) ? 0 : metok_prefill_prune_batched_workspace_bytes(static_cast<int>(B), S, Hq, Hkv, dh, Tq, n_vis, dt));
        const bool in_place = a[11] == a[0];
        const int64_t keep_stride = given(a[15]) ? integer(a[15]) : most;
        const int64_t row_stride = given(a[16]) ? integer(a[16]) : (in_place ? S : S - n_vis + most);
        const at::Tensor kept = out.get("kept_idx", {B, keep_stride}, at::kInt);
        at::Tensor hidden_out;
        PyObject* ho = given(a[11]) ? a[11] : out.find("hidden_out");
        if (ho) {
            hidden_out = tensor(ho);
            need(hidden_out.dim() == 3 && hidden_out.size(0) == B && hidden_out.size(1) == row_stride && hidden_out.size(2) == D && hidden_out.scalar_type() == hidden.scalar_type());
        } else {
            hidden_out = out.fresh({B, row_stride, D}, hidden.scalar_type());
        }
        const at::Tensor seg_out = out.get("token_seg_out", {B, keep_stride}, at::kInt);
        at::Tensor event_out, orig_out;
        if (event.defined()) event_out = out.get("token_event_out", {B, keep_stride}, at::kInt);
        if (PyObject* v = out.find("orig_idx_out")) {              // may be wider than the other lists
            orig_out = tensor(v);
            need(orig_out.scalar_type() == at::kInt && orig_out.dim() == 2 && orig_out.size(0) == B);
        } else {
            orig_out = out.fresh({B, keep_stride}, at::kInt);
        }
        auto at_ = [](const at::Tensor& t) -> void* { return t.defined() ? address(t) : nullptr; };
        Result r;
        r.put("scores", scores); r.put("kept_idx", kept);
        if (ho) { Py_INCREF(ho); r.put("hidden_out", ho); } else r.put("hidden_out", hidden_out);
        r.put("token_seg_out", seg_out); r.put("orig_idx_out", orig_out);
        Owned list(PyList_New(static_cast<Py_ssize_t>(B)));
        for (int64_t b = 0; b < B; ++b) PyList_SET_ITEM(list.o, b, Owned(PyLong_FromLongLong(keep[b])).release());
        r.put("n_keep", list.release());
        if (event_out.defined()) r.put("token_event_out", event_out);
        void* stream = stream_of(a[17]);
        return answer(launch(bound(&metok_prefill_prune_batched, static_cast<int>(B), address(hidden), S, static_cast<int>(D), dt, at_(q), at_(keys), Hq, Hkv, dh, Tq, mode,
                                   vis_start, n_vis, static_cast<const int32_t*>(address(seg)), static_cast<const int32_t*>(at_(event)), static_cast<const float*>(at_(weight)),
                                   weight.defined() ? static_cast<int>(weight.size(1)) : 0, n_seg, quota.data(), static_cast<const int32_t*>(at_(orig)),
                                   orig.defined() ? orig.size(1) : int64_t{0}, static_cast<float*>(address(scores)), static_cast<int32_t*>(address(kept)), keep_stride,
                                   address(hidden_out), row_stride, static_cast<int32_t*>(address(seg_out)), static_cast<int32_t*>(at_(event_out)),
                                   static_cast<int32_t*>(address(orig_out)), orig_out.size(1), address(ws), static_cast<size_t>(ws.numel()), stream)), r);
    });
}

// ---- stage 3 -----------------------------------------------------------------------------------------------------------
// The per-layer buffers (all of the first one's shape) and index lists of a cache.
struct Layers {
    std::vector<void*> k, v;
    std::vector<const int32_t*> idx;
    std::vector<int32_t> n_keep;
    at::Tensor first;
    int L = 0, dt = 0;

    Layers(PyObject* ks, PyObject* vs) {
        need((PyList_CheckExact(ks) || PyTuple_CheckExact(ks)) && (PyList_CheckExact(vs) || PyTuple_CheckExact(vs)));
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(ks);
        need(n >= 1 && n <= METOK_MAX_LAYERS && PySequence_Fast_GET_SIZE(vs) == n);
        L = static_cast<int>(n);
        first = tensor(PySequence_Fast_ITEMS(ks)[0]);
        need(first.dim() == 4);
        for (int i = 0; i < 4; ++i) need(first.size(i) <= INT32_MAX);
        dt = dtype_code(first);
        for (int side = 0; side < 2; ++side) {
            PyObject** items = PySequence_Fast_ITEMS(side ? vs : ks);
            for (int l = 0; l < L; ++l) {
                const at::Tensor& t = tensor(items[l]);
                need(t.sizes() == first.sizes());
                (side ? v : k).push_back(address(t));
            }
        }
    }
    void lists(PyObject* o, int64_t B) {
        need((PyList_CheckExact(o) || PyTuple_CheckExact(o)) && PySequence_Fast_GET_SIZE(o) == L);
        for (int l = 0; l < L; ++l) {
            PyObject* e = PySequence_Fast_ITEMS(o)[l];
            if (!given(e)) { idx.push_back(nullptr); n_keep.push_back(0); continue; }
            const at::Tensor& t = tensor(e);
            need(t.scalar_type() == at::kInt && t.dim() == 2 && t.size(0) == B && t.numel() > 0 && t.size(1) <= INT32_MAX);
            idx.push_back(static_cast<const int32_t*>(address(t)));
            n_keep.push_back(static_cast<int32_t>(t.size(1)));
        }
    }
};

// k_layers, v_layers, page_table (None: dense), idx, new_len, workspace, stream
PyObject* kv_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 7, [&](Launch& launch) -> PyObject* {
        Layers x(a[0], a[1]);
        const bool paged = given(a[2]);
        at::Tensor table;
        if (paged) {
            table = tensor(a[2]);
            need(table.scalar_type() == at::kInt && table.dim() == 2 && table.size(0) <= INT32_MAX && table.size(1) <= INT32_MAX);
        }
        const int64_t B = paged ? table.size(0) : x.first.size(0), Hkv = x.first.size(1), rows = x.first.size(2), dh = x.first.size(3);
        x.lists(a[3], B);
        const Outputs out(Py_None, x.first);
        at::Tensor len = given(a[4]) ? tensor(a[4]) : out.fresh({x.L}, at::kInt);
        const int64_t cap = paged ? table.size(1) * rows : rows;
        const at::Tensor ws = workspace_of(a[5], out, given(a[5]) ? 0 : metok_kv_compact_workspace_bytes(x.L, static_cast<int>(B), static_cast<int>(Hkv), cap, static_cast<int>(dh), x.dt));
        if (given(a[4])) Py_INCREF(a[4]);
        Owned result(given(a[4]) ? a[4] : THPVariable_Wrap(len));
        void* stream = stream_of(a[6]);
        auto call = [&](auto f, auto... middle) {
            return bound(f, x.k.data(), x.v.data(), x.L, static_cast<int>(B), static_cast<int>(Hkv), middle..., x.idx.data(), x.n_keep.data(),
                         static_cast<int32_t*>(address(len)), address(ws), static_cast<size_t>(ws.numel()), stream);
        };
        return answer(paged ? launch(call(&metok_kv_compact_paged, x.first.size(0), static_cast<int>(rows), static_cast<int>(dh), x.dt,
                                          static_cast<const int32_t*>(address(table)), static_cast<int>(table.size(1))))
                            : launch(call(&metok_kv_compact, rows, static_cast<int>(dh), x.dt)), result);
    });
}

// k_pools, v_pools, page_table, idx, len_in, workspace, stream
PyObject* kv_relink_paged(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 7, [&](Launch& launch) -> PyObject* {
        Layers x(a[0], a[1]);
        const at::Tensor& table = tensor(a[2]);
        need(table.scalar_type() == at::kInt && (table.dim() == 2 || (table.dim() == 3 && table.size(0) == x.L)));
        const int64_t B = table.size(-2), pages = table.size(-1), L = x.L;
        need(B <= INT32_MAX && pages <= INT32_MAX);
        x.lists(a[3], B);
        std::vector<int32_t> lens;
        if (given(a[4])) {
            quotas_of(a[4], lens);
            need(static_cast<int64_t>(lens.size()) == L);
        }
        const Outputs out(Py_None, x.first);
        const at::Tensor table_out = out.fresh({L, B, pages}, at::kInt), free_pages = out.fresh({L, B, pages}, at::kInt), n_free = out.fresh({L, B}, at::kInt),
                         copied = out.fresh({L, B}, at::kInt), len = out.fresh({L}, at::kInt);
        const int Hkv = static_cast<int>(x.first.size(1)), ps = static_cast<int>(x.first.size(2)), dh = static_cast<int>(x.first.size(3));
        const at::Tensor ws = workspace_of(a[5], out, given(a[5]) ? 0 : metok_kv_relink_paged_workspace_bytes(x.L, static_cast<int>(B), Hkv, ps, static_cast<int>(pages), dh, x.dt));
        Result r;
        r.put("page_table_out", table_out); r.put("free_pages", free_pages); r.put("n_free", n_free); r.put("rows_copied", copied); r.put("new_len", len);
        if (given(a[5])) { Py_INCREF(a[5]); r.put("workspace", a[5]); } else r.put("workspace", ws);
        void* stream = stream_of(a[6]);
        return answer(launch(bound(&metok_kv_relink_paged, x.k.data(), x.v.data(), x.L, static_cast<int>(B), Hkv, x.first.size(0), ps, dh, x.dt,
                                   static_cast<const int32_t*>(address(table)), table.dim() == 2 ? int64_t{0} : B * pages, static_cast<int>(pages),
                                   given(a[4]) ? lens.data() : nullptr, x.idx.data(), x.n_keep.data(), static_cast<int32_t*>(address(table_out)),
                                   static_cast<int32_t*>(address(free_pages)), static_cast<int32_t*>(address(n_free)), static_cast<int32_t*>(address(copied)),
                                   static_cast<int32_t*>(address(len)), address(ws), static_cast<size_t>(ws.numel()), stream)), r);
    });
}

// ---- decoding ----------------------------------------------------------------------------------------------------------
// A tensor of this type, shape and place.
inline const at::Tensor& fitting(PyObject* o, at::ScalarType type, at::IntArrayRef shape, const at::Tensor& like) {
    const at::Tensor& t = tensor(o);
    need(t.scalar_type() == type && t.sizes() == shape && t.device() == like.device());
    return t;
}
inline const at::Tensor& beside(const at::Tensor& t, const at::Tensor& like) { need(t.device() == like.device()); return t; }

// q, k, v, page_table (None: dense), lens, k_new, v_new, scale, logit_cap, weight, workspace, out, stream; FOUR: over a cache in 4 bits
template <bool FOUR>
PyObject* decode_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 13, [&](Launch& launch) -> PyObject* {
        const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]);
        need(q.dim() == 3 && k.dim() == 4);
        const auto type = q.scalar_type();
        const int dt = dtype_code(q);
        const auto held = FOUR ? at::kByte : type;
        const int64_t B = q.size(0), Hq = q.size(1), dh = q.size(2), Hkv = k.size(1);
        need(B <= INT32_MAX && Hq <= INT32_MAX && dh <= INT32_MAX && Hkv <= INT32_MAX && k.size(2) < INT32_MAX / (FOUR ? 16 : 1));
        const int64_t rows = k.size(2) * (FOUR ? 16 : 1);
        need(k.scalar_type() == held && k.size(3) == (FOUR ? 17 * dh / 2 : dh) && k.device() == q.device());
        const at::Tensor& v = fitting(a[2], held, k.sizes(), q);
        const bool paged = given(a[3]);
        at::Tensor table;
        int64_t cap = rows;
        if (paged) {
            table = beside(tensor(a[3]), q);
            need(table.scalar_type() == at::kInt && table.dim() == 2 && table.size(0) == B && table.size(1) <= INT32_MAX);
            cap = table.size(1) * rows;
        } else {
            need(k.size(0) == B);
        }
        const at::Tensor& lens = fitting(a[4], at::kInt, {B}, q);
        need(given(a[5]) == given(a[6]));
        void *k_new = nullptr, *v_new = nullptr;
        if (given(a[5])) {
            k_new = address(fitting(a[5], type, {B, Hkv, dh}, q));
            v_new = address(fitting(a[6], type, {B, Hkv, dh}, q));
        }
        const double scale = given(a[7]) ? real(a[7]) : 1.0 / std::sqrt(static_cast<double>(dh)), logit_cap = real(a[8]);
        at::Tensor weight;
        if (given(a[9])) {
            weight = beside(tensor(a[9]), q);
            need(weight.scalar_type() == at::kFloat && weight.dim() == 2 && weight.size(0) == B);
        }
        const Outputs out(a[11], q);
        const at::Tensor result = beside(out.get("out", {B, Hq, dh}, type), q), lse = beside(out.get("lse", {B, Hq}, at::kFloat), q);
        const at::Tensor ws = beside(workspace_of(a[10], out, given(a[10]) ? 0 : (FOUR ? metok_kv4_attention_workspace_bytes : metok_decode_attention_workspace_bytes)(
            static_cast<int>(B), static_cast<int>(Hq), static_cast<int>(Hkv), cap, static_cast<int>(dh), dt, weight.defined())), q);
        Result r;
        r.put("out", result); r.put("lse", lse);
        void* stream = stream_on(a[12], q);
        float* w = weight.defined() ? static_cast<float*>(address(weight)) : nullptr;
        const int64_t w_stride = weight.defined() ? weight.size(1) : 0;
        auto call = [&](auto f, auto... middle) {
            return bound(f, address(q), static_cast<int>(B), static_cast<int>(Hq), static_cast<int>(Hkv), static_cast<int>(dh), dt, address(k), address(v), middle...,
                         static_cast<const int32_t*>(address(lens)), k_new, v_new, scale, logit_cap, address(result), static_cast<float*>(address(lse)), w, w_stride,
                         address(ws), static_cast<size_t>(ws.nbytes()), stream);
        };
        return answer(paged ? launch(call(FOUR ? &metok_kv4_attention_paged : &metok_decode_attention_paged, k.size(0), static_cast<int>(rows), static_cast<const int32_t*>(address(table)),
                                          static_cast<int>(table.size(1))))
                            : launch(call(FOUR ? &metok_kv4_attention : &metok_decode_attention, rows)), r);
    });
}

// ---- queries, keys and values of new tokens ----------------------------------------------------------------------------
// An int32 per video, or NULL.
inline const int32_t* per_video(PyObject* o, int64_t B, const at::Tensor& like) {
    return given(o) ? static_cast<const int32_t*>(address(fitting(o, at::kInt, {B}, like))) : nullptr;
}
// The page table of a paged call.  One without columns has no address, and the call that it belongs to is a paged one all the same, which the library refuses.
struct Table {
    const bool paged;
    const int32_t* p = nullptr;
    int per_seq = 0;
    Table(PyObject* o, int64_t B, const at::Tensor& like) : paged(given(o)) {
        if (!paged) return;
        const at::Tensor& t = beside(tensor(o), like);
        need(t.scalar_type() == at::kInt && t.dim() == 2 && t.size(0) == B && t.size(1) <= INT32_MAX);
        p = static_cast<const int32_t*>(address(t));
        per_seq = static_cast<int>(t.size(1));
    }
};
// Rows of tokens [B, n, heads, dh] that may be parts of a wider buffer: elements between tokens.
struct TokenRows {
    void* p;
    int heads;
    int64_t stride;
    TokenRows(PyObject* o, const at::Tensor& like) {
        need(THPVariable_CheckExact(o));
        const at::Tensor& t = THPVariable_Unpack(o);
        need(t.is_cuda() && t.layout() == at::kStrided && t.dim() == 4 && t.scalar_type() == like.scalar_type() && t.device() == like.device() &&
             t.size(0) == like.size(0) && t.size(1) == like.size(1) && t.size(3) == like.size(3) && t.size(2) <= INT32_MAX && t.numel() > 0);
        const int64_t B = t.size(0), n = t.size(1), dh = t.size(3);
        heads = static_cast<int>(t.size(2));
        stride = n > 1 ? t.stride(1) : B > 1 ? t.stride(0) : heads * dh;
        need((t.stride(3) == 1) && (heads == 1 || t.stride(2) == dh) && (B == 1 || t.stride(0) == n * stride));
        p = address(t);
    }
};

// q, k, v, pos, inv_freq, k_cache, v_cache, page_table (None: dense), start, count, pair_axis, q_weight, k_weight, eps, pairs, out, stream
PyObject* rotate_qk(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded(n_args, 17, [&](Launch& launch) -> PyObject* {
        need(THPVariable_CheckExact(a[0]));
        const at::Tensor& like = THPVariable_Unpack(a[0]);
        need(like.is_cuda() && like.dim() == 4 && like.size(0) <= INT32_MAX && like.size(3) <= INT32_MAX);
        const auto type = like.scalar_type();
        const int dt = dtype_code(like);
        const int64_t B = like.size(0), n = like.size(1), dh = like.size(3);
        const TokenRows q(a[0], like), k(a[1], like), v(a[2], like);
        need(k.heads == v.heads);
        const at::Tensor& k_to = beside(tensor(a[5]), like);
        need(k_to.dim() == 4 && k_to.scalar_type() == type && k_to.size(1) == k.heads && k_to.size(3) == dh && k_to.size(2) <= INT32_MAX);
        const at::Tensor& v_to = fitting(a[6], type, k_to.sizes(), like);
        const Table table(a[7], B, like);
        need(table.paged || k_to.size(0) == B);
        const at::Tensor &pos = beside(tensor(a[3]), like), &freq = beside(tensor(a[4]), like);
        need(pos.scalar_type() == at::kInt && (pos.dim() == 3 || pos.dim() == 2) && pos.size(-2) == B && pos.size(-1) == n && freq.scalar_type() == at::kFloat && freq.dim() == 1);
        const int64_t axes = pos.dim() == 3 ? pos.size(0) : 1, half = freq.size(0);
        need(axes <= INT32_MAX && half <= 1024);
        const uint8_t* axis = nullptr;
        if (given(a[10])) {
            need(PyBytes_CheckExact(a[10]) && PyBytes_GET_SIZE(a[10]) == half);
            axis = reinterpret_cast<const uint8_t*>(PyBytes_AS_STRING(a[10]));
        }
        auto weight = [&](PyObject* o) { return given(o) ? address(fitting(o, type, {dh}, like)) : nullptr; };
        void *q_weight = weight(a[11]), *k_weight = weight(a[12]);
        const double eps = real(a[13]);
        const int pairs = int32(a[14]);
        const int32_t *start = per_video(a[8], B, like), *count = per_video(a[9], B, like);
        const Outputs out(a[15], like);
        const at::Tensor to = beside(out.get("q", {B, q.heads, n, dh}, type), like);
        Result r;
        r.put("q", to);
        void* stream = stream_on(a[16], like);
        auto call = [&](auto f, auto... tail) {
            return bound(f, q.p, k.p, v.p, q.stride, k.stride, v.stride, static_cast<int>(B), n, q.heads, k.heads, static_cast<int>(dh), dt, count, q_weight, k_weight, eps,
                         static_cast<const int32_t*>(address(pos)), static_cast<int>(axes), static_cast<const float*>(address(freq)), axis, static_cast<int>(2 * half), pairs,
                         address(to), address(k_to), address(v_to), tail..., start, stream);
        };
        return answer(table.paged ? launch(call(&metok_rotate_qk_paged, k_to.size(0), static_cast<int>(k_to.size(2)), table.p, table.per_seq))
                              : launch(call(&metok_rotate_qk, k_to.size(2))), r);
    });
}

// A cache in 4 bits or its pools: [slabs, Hkv, rows / 16, 17 dh / 2] bytes.
struct Cache4 {
    const at::Tensor &k, &v;
    int64_t slabs, rows;
    int Hkv, dh;
    Cache4(PyObject* ko, PyObject* vo, const at::Tensor& like) : k(beside(tensor(ko), like)), v(fitting(vo, at::kByte, k.sizes(), like)) {
        need(k.scalar_type() == at::kByte && k.dim() == 4 && k.size(1) <= INT32_MAX && k.size(2) < INT32_MAX / 16 && k.size(3) <= INT32_MAX / 2);
        slabs = k.size(0);
        Hkv = static_cast<int>(k.size(1));
        rows = 16 * k.size(2);
        dh = static_cast<int>(k.size(3) * 2 / 17);
        need(17 * dh / 2 == k.size(3));
    }
};

// k, v, k_cache, v_cache, page_table (None: dense), start, count, idx, stream
PyObject* kv4_pack(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded(n_args, 9, [&](Launch& launch) -> PyObject* {
        const at::Tensor& k = tensor(a[0]);
        const int dt = dtype_code(k);
        need(k.dim() == 4 && k.size(0) <= INT32_MAX);
        const at::Tensor& v = fitting(a[1], k.scalar_type(), k.sizes(), k);
        const Cache4 to(a[2], a[3], k);
        const int64_t B = k.size(0);
        need(to.Hkv == k.size(1) && to.dh == k.size(3));
        const Table table(a[4], B, k);
        need(table.paged || to.slabs == B);
        const int32_t *start = per_video(a[5], B, k), *count = per_video(a[6], B, k), *idx = nullptr;
        int64_t n = k.size(2);
        if (given(a[7])) {
            const at::Tensor& t = beside(tensor(a[7]), k);
            need(t.scalar_type() == at::kInt && t.dim() == 2 && t.size(0) == B);
            idx = static_cast<const int32_t*>(address(t));
            n = t.size(1);
        }
        Owned done(PyLong_FromLong(METOK_OK));
        void* stream = stream_on(a[8], k);
        auto call = [&](auto f, auto... tail) {
            return bound(f, address(k), address(v), static_cast<int>(B), to.Hkv, k.size(2), to.dh, dt, idx, n, count, address(to.k), address(to.v), tail..., start, stream);
        };
        return answer(table.paged ? launch(call(&metok_kv4_pack_paged, to.slabs, static_cast<int>(to.rows), table.p, table.per_seq)) : launch(call(&metok_kv4_pack, to.rows)), done);
    });
}

// k_cache, v_cache, page_table (None: dense), lens, n, first, idx, out, stream; both outputs are given
PyObject* kv4_unpack(PyObject*, PyObject* const* a, Py_ssize_t n_args) {
    return guarded(n_args, 9, [&](Launch& launch) -> PyObject* {
        const Cache4 from(a[0], a[1], tensor(a[0]));
        const at::Tensor& lens = beside(tensor(a[3]), from.k);
        need(lens.scalar_type() == at::kInt && lens.dim() == 1 && lens.size(0) <= INT32_MAX);
        const int64_t B = lens.size(0), n = integer(a[4]);
        const Table table(a[2], B, from.k);
        need(table.paged || from.slabs == B);
        const Outputs out(a[7], from.k);
        PyObject *ko = out.find("k"), *vo = out.find("v");
        need(ko && vo);
        const at::Tensor& k = beside(tensor(ko), from.k);
        const int dt = dtype_code(k);
        need(k.dim() == 4 && k.size(0) == B && k.size(1) == from.Hkv && k.size(3) == from.dh);
        const at::Tensor& v = fitting(vo, k.scalar_type(), k.sizes(), k);
        const int32_t *first = per_video(a[5], B, from.k), *idx = given(a[6]) ? static_cast<const int32_t*>(address(fitting(a[6], at::kInt, {B, n}, from.k))) : nullptr;
        Result r;
        r.put("k", k); r.put("v", v);
        void* stream = stream_on(a[8], from.k);
        auto call = [&](auto f, auto... middle) {
            return bound(f, address(from.k), address(from.v), static_cast<int>(B), from.Hkv, middle..., static_cast<const int32_t*>(address(lens)), first, idx, n,
                         address(k), address(v), k.size(2), dt, stream);
        };
        return answer(table.paged ? launch(call(&metok_kv4_unpack_paged, from.slabs, static_cast<int>(from.rows), from.dh, table.p, table.per_seq))
                              : launch(call(&metok_kv4_unpack, from.rows, from.dh)), r);
    });
}

// What the eviction calls share: weight, lens, budget, n_first, n_last, weight_out, idx, new_len.
struct Eviction {
    std::vector<const float*> weight;
    std::vector<float*> weight_out;
    std::vector<int32_t*> idx;
    std::vector<int32_t> budget;
    at::Tensor first, lens, new_len;
    int64_t B = 0, W = 0;
    int L = 0, n_first = 0, n_last = 0;
    Result result;

    static PyObject** items(PyObject* o, Py_ssize_t n) {
        need((PyList_CheckExact(o) || PyTuple_CheckExact(o)) && PySequence_Fast_GET_SIZE(o) == n);
        return PySequence_Fast_ITEMS(o);
    }
    explicit Eviction(PyObject* const* a) {
        need(PyList_CheckExact(a[0]) || PyTuple_CheckExact(a[0]));
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(a[0]);
        need(n >= 1 && n <= METOK_MAX_LAYERS);
        L = static_cast<int>(n);
        PyObject **w = items(a[0], n), **to = given(a[5]) ? items(a[5], n) : w, **lists = given(a[6]) ? items(a[6], n) : nullptr;
        for (int l = 0; l < L && !first.defined(); ++l)
            if (given(w[l])) first = tensor(w[l]);
        need(first.defined() && first.scalar_type() == at::kFloat && first.dim() == 2);
        B = first.size(0); W = first.size(1);
        need(B <= INT32_MAX);
        if (PyLong_CheckExact(a[2])) budget.assign(static_cast<size_t>(L), int32(a[2]));
        else {
            PyObject** each = items(a[2], n);
            for (int l = 0; l < L; ++l) budget.push_back(int32(each[l]));
        }
        n_first = int32(a[3]); n_last = int32(a[4]);
        lens = fitting(a[1], at::kInt, {L, B}, first);
        const Outputs fresh(Py_None, first);
        Owned made(PyList_New(L)), moved(PyList_New(L));
        auto place = [](const Owned& list, int l, PyObject* o) { PyList_SET_ITEM(list.o, l, o); };         // takes the reference
        for (int l = 0; l < L; ++l) {
            Py_INCREF(to[l]);
            place(moved, l, to[l]);
            if (!given(w[l])) {
                weight.push_back(nullptr); weight_out.push_back(nullptr); idx.push_back(nullptr);
                Py_INCREF(Py_None);
                place(made, l, Py_None);
                continue;
            }
            need(budget[l] >= 0);
            weight.push_back(static_cast<const float*>(address(fitting(w[l], at::kFloat, {B, W}, first))));
            weight_out.push_back(static_cast<float*>(address(fitting(to[l], at::kFloat, {B, W}, first))));
            if (lists && given(lists[l])) {
                idx.push_back(static_cast<int32_t*>(address(fitting(lists[l], at::kInt, {B, budget[l]}, first))));
                Py_INCREF(lists[l]);
                place(made, l, lists[l]);
            } else {
                const at::Tensor t = fresh.fresh({B, budget[l]}, at::kInt);
                idx.push_back(static_cast<int32_t*>(address(t)));
                place(made, l, Owned(THPVariable_Wrap(t)).release());
            }
        }
        new_len = given(a[7]) ? fitting(a[7], at::kInt, {L, B}, first) : fresh.fresh({L, B}, at::kInt);
        result.put("idx", made.release());
        if (given(a[7])) { Py_INCREF(a[7]); result.put("new_len", a[7]); } else result.put("new_len", new_len);
        result.put("weight", moved.release());
    }
    const int32_t* lengths() const { return static_cast<const int32_t*>(address(lens)); }
    int32_t* lengths_out() const { return static_cast<int32_t*>(address(new_len)); }
};

// weight, lens, budget, n_first, n_last, weight_out, idx, new_len, k_layers, v_layers, page_table (None: dense), workspace, stream
PyObject* kv_evict(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 13, [&](Launch& launch) -> PyObject* {
        Eviction e(a);
        const Layers x(a[8], a[9]);
        need(x.L == e.L);
        for (int side = 8; side < 10; ++side)
            for (int l = 0; l < x.L; ++l) {
                const at::Tensor& t = THPVariable_Unpack(PySequence_Fast_ITEMS(a[side])[l]);
                need(t.device() == e.first.device() && t.scalar_type() == x.first.scalar_type());
            }
        const bool paged = given(a[10]);
        const int Hkv = static_cast<int>(x.first.size(1)), dh = static_cast<int>(x.first.size(3)), B = static_cast<int>(e.B);
        const int64_t rows = x.first.size(2);
        at::Tensor table;
        if (paged) {
            table = beside(tensor(a[10]), e.first);
            need(table.scalar_type() == at::kInt && table.dim() == 2 && table.size(0) == e.B && table.size(1) <= INT32_MAX);
        } else {
            need(x.first.size(0) == e.B);
        }
        const int64_t cap = paged ? table.size(1) * rows : rows;
        const Outputs out(Py_None, e.first);
        const at::Tensor ws = beside(workspace_of(a[11], out, given(a[11]) ? 0 : metok_kv_evict_workspace_bytes(x.L, B, Hkv, cap, dh, x.dt)), e.first);
        void* stream = stream_on(a[12], e.first);
        auto call = [&](auto f, auto... middle) {
            return bound(f, x.k.data(), x.v.data(), x.L, B, Hkv, middle..., e.weight.data(), e.weight_out.data(), e.W, e.lengths(), e.budget.data(), e.n_first, e.n_last,
                         e.idx.data(), e.lengths_out(), address(ws), static_cast<size_t>(ws.nbytes()), stream);
        };
        return answer(paged ? launch(call(&metok_kv_evict_paged, x.first.size(0), static_cast<int>(rows), dh, x.dt, static_cast<const int32_t*>(address(table)),
                                          static_cast<int>(table.size(1))))
                            : launch(call(&metok_kv_evict, rows, dh, x.dt)), e.result);
    });
}

// weight, lens, budget, n_first, n_last, weight_out, idx, new_len, S_cap, stream
PyObject* kv_evict_select(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(n, 10, [&](Launch& launch) -> PyObject* {
        Eviction e(a);
        const int64_t S_cap = integer(a[8]);
        void* stream = stream_on(a[9], e.first);
        return answer(launch(bound(&metok_kv_evict_select, e.weight.data(), e.weight_out.data(), e.W, e.L, static_cast<int>(e.B), S_cap, e.lengths(), e.budget.data(),
                                   e.n_first, e.n_last, e.idx.data(), e.lengths_out(), stream)), e.result);
    });
}

#define METOK_HOST_CALL(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL, nullptr
PyMethodDef methods[] = {
    {"segment_compress", METOK_HOST_CALL(&segment_compress<false>)},
    {"segment_compress_batched", METOK_HOST_CALL(&segment_compress<true>)},
    {"prefill_prune", METOK_HOST_CALL(&prefill_prune)},
    {"prefill_prune_batched", METOK_HOST_CALL(&prefill_prune_batched)},
    {"kv_compact", METOK_HOST_CALL(&kv_compact)},
    {"kv_relink_paged", METOK_HOST_CALL(&kv_relink_paged)},
    {"decode_attention", METOK_HOST_CALL(&decode_attention<false>)},
    {"kv4_attention", METOK_HOST_CALL(&decode_attention<true>)},
    {"rotate_qk", METOK_HOST_CALL(&rotate_qk)},
    {"kv4_pack", METOK_HOST_CALL(&kv4_pack)},
    {"kv4_unpack", METOK_HOST_CALL(&kv4_unpack)},
    {"kv_evict", METOK_HOST_CALL(&kv_evict)},
    {"kv_evict_select", METOK_HOST_CALL(&kv_evict_select)},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// The tensors' layout is that of the torch whose headers this was built with.
PyMODINIT_FUNC PyInit__host() {
    try {
        const Owned torch(PyImport_ImportModule("torch")), version(PyObject_GetAttrString(torch.o, "__version__"));
        const Owned text(PyObject_Str(version.o));
        if (PyUnicode_CompareWithASCIIString(text.o, METOK_TORCH_VERSION) != 0) {
            PyErr_Format(PyExc_ImportError, "built for torch %s, this is %U", METOK_TORCH_VERSION, text.o);
            return nullptr;
        }
    } catch (const Raised&) {
        return nullptr;
    }
    return PyModule_Create(&module);
}
