// The serving operators' Python calls on torch tensors, without the interpreter's share of the time: types, shapes, strides
// and devices of the tensors are checked and the C functions called, in well under a microsecond.  A CPython module; the
// C library itself knows nothing of torch.
//
// Every function returns the C status, or a text that says which tensor does not fit.  Tensors on the host are checked like those
// on a GPU, and refused last.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "amoeba.h"

namespace {

struct Refused {
    const char* why;
};

template <class T>
const T* at_address(PyObject* o) {
    return o == Py_None ? nullptr : static_cast<const T*>(PyLong_AsVoidPtr(o));
}
int64_t whole(PyObject* o) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused{nullptr};
    return v;
}
int32_t whole32(PyObject* o) {
    const int64_t v = whole(o);
    if (v < INT32_MIN || v > INT32_MAX) throw Refused{"a number does not fit 32 bits"};
    return (int32_t)v;
}
double real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1. && PyErr_Occurred()) throw Refused{nullptr};
    return v;
}
const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) throw Refused{"a tensor is needed"};
    return THPVariable_Unpack(o);
}
// device: of a GPU, or -1 for the host.
bool on(const at::Tensor& t, int64_t device) { return device < 0 ? t.is_cpu() : t.is_cuda() && t.device().index() == device; }

// Address of a dense tensor with at least n elements.
void* dense(PyObject* o, at::ScalarType type, int64_t n, int64_t device, const char* why) {
    const at::Tensor& t = tensor(o);
    if (t.scalar_type() != type || !on(t, device) || !t.is_contiguous() || t.numel() < n) throw Refused{why};
    return t.data_ptr();
}

struct Pointers {
    void* p[AMOEBA_MAX_TP];
    int64_t stride = 0;
    operator void**() { return p; }
};
// The tensors of a list or tuple, one per worker.
PyObject** workers(PyObject* list, int32_t tp, const char* why) {
    if (!PyList_Check(list) && !PyTuple_Check(list)) throw Refused{"one tensor per worker is needed, as a list or tuple"};
    if (tp < 1 || tp > AMOEBA_MAX_TP || PySequence_Fast_GET_SIZE(list) != tp) throw Refused{why};
    return PySequence_Fast_ITEMS(list);
}
void pools(PyObject* list, const amoeba_layout& l, int64_t bytes, bool scores, int64_t device, Pointers* out) {
    PyObject** items = workers(list, l.tp, scores ? "score pool count != tp" : "pool count != tp");
    for (int r = 0; r < l.tp; ++r) {
        const at::Tensor& t = tensor(items[r]);
        if (scores && t.scalar_type() != at::kFloat) throw Refused{"score pools are float32"};
        if (!on(t, device) || !t.is_contiguous() || (int64_t)t.nbytes() < bytes)
            throw Refused{"a pool is on another device, strided or too small"};
        out->p[r] = t.data_ptr();
    }
}
// [>= rows, width] or [>= rows, heads, head_dim] row buffers, dense along a row, equally strided; rows may not overlap (a
// broadcast row has stride 0, which means dense rows to the C call).  A tensor of one row fits beside any stride.
void rows(PyObject* list, const amoeba_layout& l, int64_t n_rows, int64_t width, at::ScalarType type, int64_t device, Pointers* out) {
    static const char* why =
        "row buffers are [>= num_rows, heads of the worker * head_dim] of the element type, on the batch's device, dense along a "
        "row, equally strided and without rows that overlap";
    PyObject** items = workers(list, l.tp, "row buffer count != tp");
    out->stride = 0;
    for (int r = 0; r < l.tp; ++r) {
        const at::Tensor& t = tensor(items[r]);
        const int64_t dim = t.dim();
        if (t.scalar_type() != type || !on(t, device) || (dim != 2 && dim != 3) || t.size(0) < n_rows || t.stride(dim - 1) != 1)
            throw Refused{why};
        if (dim == 3 ? t.size(1) * t.size(2) != width || (t.size(1) > 1 && t.stride(1) != t.size(2)) : t.size(1) != width)
            throw Refused{why};
        if (t.size(0) > 1) {
            if (t.stride(0) < width || (out->stride && t.stride(0) != out->stride)) throw Refused{why};
            out->stride = t.stride(0);
        }
        out->p[r] = t.data_ptr();
    }
}

at::ScalarType element(int32_t dtype) {
    if (dtype == AMOEBA_FP16) return at::kHalf;
    if (dtype == AMOEBA_BF16) return at::kBFloat16;
    throw Refused{"dtype is DTYPE_FP16 or DTYPE_BF16"};
}
int64_t layer_bytes(const amoeba_layout& l) {
    const amoeba_model& m = l.model;
    return l.kv_layer_stride_bytes ? l.kv_layer_stride_bytes
                                   : (int64_t)l.num_blocks * (m.num_kv_heads / l.tp) * 2 * l.block_tokens * m.head_dim * m.elem_bytes;
}
int64_t layer_scores(const amoeba_layout& l) {
    return (int64_t)l.num_blocks * (l.model.num_kv_heads / l.tp) * l.block_tokens * 4;
}
const amoeba_layout& layout_of(PyObject* o) {
    const amoeba_layout* l = at_address<amoeba_layout>(o);
    if (!l || l->tp < 1 || l->tp > AMOEBA_MAX_TP) throw Refused{"the layout's tp"};
    return *l;
}
// The stream to launch on, with its device current while the object lives.
struct On {
    void* stream;
    c10::cuda::CUDAGuard guard;
    static c10::DeviceIndex gpu(int64_t device) {
        if (device < 0) throw Refused{"the tensors are not on a GPU"};
        return (c10::DeviceIndex)device;
    }
    static void* handle(PyObject* o) {
        void* p = o == Py_None ? nullptr : PyLong_AsVoidPtr(o);
        if (!p && PyErr_Occurred()) throw Refused{nullptr};
        return p;
    }
    On(int64_t device, PyObject* given) : stream(handle(given)), guard(gpu(device)) {
        if (given == Py_None) stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    }
};

template <class F>
PyObject* answer(Py_ssize_t given, Py_ssize_t wanted, F call) {
    if (given != wanted) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        return PyLong_FromLong((long)call());
    } catch (const Refused& r) {
        if (PyErr_Occurred()) return nullptr;
        return PyUnicode_FromString(r.why ? r.why : "bad number");
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// (layout, dtype, layer, pools, batch, device, q, k, v, rotation, q_out, status, stream)
PyObject* append_kv(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return answer(n, 13, [&] {
        const amoeba_layout& l = layout_of(a[0]);
        const int32_t dtype = whole32(a[1]), layer = whole32(a[2]);
        const amoeba_batch* b = at_address<amoeba_batch>(a[4]);
        const int64_t dev = whole(a[5]), D = l.model.head_dim;
        const at::ScalarType type = element(dtype);
        Pointers pool, q, k, v, out;
        pools(a[3], l, layer_bytes(l) * ((int64_t)layer + 1), false, dev, &pool);
        const bool has_q = a[6] != Py_None, has_out = a[10] != Py_None;
        if (has_q) rows(a[6], l, b->num_rows, l.model.num_q_heads / l.tp * D, type, dev, &q);
        rows(a[7], l, b->num_rows, l.model.num_kv_heads / l.tp * D, type, dev, &k);
        rows(a[8], l, b->num_rows, l.model.num_kv_heads / l.tp * D, type, dev, &v);
        if (has_out) rows(a[10], l, b->num_rows, l.model.num_q_heads / l.tp * D, type, dev, &out);
        void* status = dense(a[11], at::kInt, 1, dev, "status is int32");
        const On here(dev, a[12]);
        return amoeba_append_kv(&l, dtype, layer, pool, b, has_q ? (void**)q : nullptr, q.stride, k, k.stride, v, v.stride,
                                at_address<amoeba_rotation>(a[9]), has_out ? (void**)out : nullptr, out.stride, (int32_t*)status,
                                here.stream);
    });
}
// (layout, dtype, layer, pools, batch, device, q, scale, window, out, lse, status, workspace, stream)
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return answer(n, 14, [&] {
        const amoeba_layout& l = layout_of(a[0]);
        const int32_t dtype = whole32(a[1]), layer = whole32(a[2]);
        const amoeba_batch* b = at_address<amoeba_batch>(a[4]);
        const int64_t dev = whole(a[5]), width = (int64_t)l.model.num_q_heads / l.tp * l.model.head_dim;
        const at::ScalarType type = element(dtype);
        Pointers pool, q, out;
        pools(a[3], l, layer_bytes(l) * ((int64_t)layer + 1), false, dev, &pool);
        rows(a[6], l, b->num_rows, width, type, dev, &q);
        rows(a[9], l, b->num_rows, width, type, dev, &out);
        const double scale = real(a[7]);
        const int32_t window = whole32(a[8]);
        void* lse = a[10] == Py_None ? nullptr
                                     : dense(a[10], at::kFloat, (int64_t)b->num_rows * l.model.num_q_heads, dev,
                                             "lse is float32 [num_rows, num_q_heads]");
        void* status = dense(a[11], at::kInt, 1, dev, "status is int32");
        void* ws = dense(a[12], at::kByte, 0, dev, "the workspace is uint8");
        const On here(dev, a[13]);
        return amoeba_attend(&l, dtype, layer, pool, b, q, q.stride, (float)scale, window, out, out.stride, (float*)lse,
                             (int32_t*)status, ws, tensor(a[12]).numel(), here.stream);
    });
}
// (layout, dtype, layer, pools, batch, device, q, scale, window, lse, scored_lens, score_pools, status, stream)
PyObject* accumulate_scores(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return answer(n, 14, [&] {
        const amoeba_layout& l = layout_of(a[0]);
        const int32_t dtype = whole32(a[1]), layer = whole32(a[2]);
        const amoeba_batch* b = at_address<amoeba_batch>(a[4]);
        const int64_t dev = whole(a[5]);
        const at::ScalarType type = element(dtype);
        Pointers pool, q, scores;
        pools(a[3], l, layer_bytes(l) * ((int64_t)layer + 1), false, dev, &pool);
        pools(a[11], l, layer_scores(l) * ((int64_t)layer + 1), true, dev, &scores);
        rows(a[6], l, b->num_rows, (int64_t)l.model.num_q_heads / l.tp * l.model.head_dim, type, dev, &q);
        const double scale = real(a[7]);
        const int32_t window = whole32(a[8]);
        void* lse = dense(a[9], at::kFloat, (int64_t)b->num_rows * l.model.num_q_heads, dev, "lse is float32 [num_rows, num_q_heads]");
        void* scored = a[10] == Py_None ? nullptr : dense(a[10], at::kInt, b->num_seqs, dev, "scored_lens is int32 [num_seqs]");
        void* status = dense(a[12], at::kInt, 1, dev, "status is int32");
        const On here(dev, a[13]);
        return amoeba_accumulate_scores(&l, dtype, layer, pool, b, q, q.stride, (float)scale, window, (float*)lse, (int32_t*)scored,
                                        (float* const*)scores.p, (int32_t*)status, here.stream);
    });
}
// (layout, layer_begin, layer_end, pools, score_pools, src_bt, seq_lens, dst_bt, budget, recent, new_lens, status, workspace,
//  stream)
PyObject* evict_kv(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return answer(n, 14, [&] {
        const amoeba_layout& l = layout_of(a[0]);
        const int32_t l0 = whole32(a[1]), l1 = whole32(a[2]), budget = whole32(a[8]), recent = whole32(a[9]);
        const at::Tensor &lens = tensor(a[6]), &src = tensor(a[5]), &dst = tensor(a[7]);
        const int64_t dev = lens.is_cuda() ? lens.device().index() : -1, S = lens.numel();
        if (src.dim() != 2 || dst.dim() != 2 || src.size(0) != S || dst.size(0) != S) throw Refused{"block tables are [num_seqs, blocks]"};
        if (S > INT32_MAX || src.size(1) > INT32_MAX || dst.size(1) > INT32_MAX) throw Refused{"too many sequences or blocks"};
        Pointers pool, scores;
        pools(a[3], l, layer_bytes(l) * l1, false, dev, &pool);
        const bool has_scores = a[4] != Py_None;
        if (has_scores) pools(a[4], l, layer_scores(l) * l1, true, dev, &scores);
        void* src_p = dense(a[5], at::kInt, 0, dev, "block tables are int32");
        void* lens_p = dense(a[6], at::kInt, S, dev, "lengths are int32");
        void* dst_p = dense(a[7], at::kInt, 0, dev, "block tables are int32");
        void* new_p = dense(a[10], at::kInt, S, dev, "lengths are int32");
        void* status = dense(a[11], at::kInt, 1, dev, "status is int32");
        void* ws = dense(a[12], at::kByte, 0, dev, "the workspace is uint8");
        const On here(dev, a[13]);
        return amoeba_evict_kv(&l, l0, l1, pool, has_scores ? (float* const*)scores.p : nullptr, (int32_t*)src_p, (int32_t*)lens_p,
                               (int32_t)S, (int32_t)src.size(1), (int32_t*)dst_p, (int32_t)dst.size(1), budget, recent,
                               (int32_t*)new_p, (int32_t*)status, ws, tensor(a[12]).numel(), here.stream);
    });
}

// (layout, dtype, layer, pools, batch, device, prefixes, prefixes' device, q, scale, out, lse, status, workspace, stream)
PyObject* attend_shared(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return answer(n, 15, [&] {
        const amoeba_layout& l = layout_of(a[0]);
        const int32_t dtype = whole32(a[1]), layer = whole32(a[2]);
        const amoeba_batch* b = at_address<amoeba_batch>(a[4]);
        const int64_t dev = whole(a[5]), width = (int64_t)l.model.num_q_heads / l.tp * l.model.head_dim;
        if (whole(a[7]) != dev) throw Refused{"the prefixes are on another device than the batch"};
        const at::ScalarType type = element(dtype);
        Pointers pool, q, out;
        pools(a[3], l, layer_bytes(l) * ((int64_t)layer + 1), false, dev, &pool);
        rows(a[8], l, b->num_rows, width, type, dev, &q);
        rows(a[10], l, b->num_rows, width, type, dev, &out);
        const double scale = real(a[9]);
        void* lse = a[11] == Py_None ? nullptr
                                     : dense(a[11], at::kFloat, (int64_t)b->num_rows * l.model.num_q_heads, dev,
                                             "lse is float32 [num_rows, num_q_heads]");
        void* status = dense(a[12], at::kInt, 1, dev, "status is int32");
        void* ws = dense(a[13], at::kByte, 0, dev, "the workspace is uint8");
        const On here(dev, a[14]);
        return amoeba_attend_shared(&l, dtype, layer, pool, b, at_address<amoeba_prefixes>(a[6]), q, q.stride, (float)scale, out,
                                    out.stride, (float*)lse, (int32_t*)status, ws, tensor(a[13]).numel(), here.stream);
    });
}
// (layout, block_table, block_refs, seq_lens, new_lens, parents, shared_lens, lens_out, q_starts, num_rows, first_positions, positions,
//  slots, pairs, num_pairs, free_count, status, stream)
PyObject* advance_tables(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return answer(n, 18, [&] {
        const amoeba_layout& l = layout_of(a[0]);
        const at::Tensor &table = tensor(a[1]), &lens = tensor(a[3]);
        const int64_t dev = lens.is_cuda() ? lens.device().index() : -1, S = lens.numel();
        if (table.dim() != 2 || table.size(0) != S) throw Refused{"block tables are [num_seqs, blocks]"};
        if (S > INT32_MAX || table.size(1) > INT32_MAX) throw Refused{"too many sequences or blocks"};
        amoeba_table_step s{};
        auto ints = [&](int i, int64_t count, const char* why) {
            return a[i] == Py_None ? nullptr : (int32_t*)dense(a[i], at::kInt, count, dev, why);
        };
        s.num_seqs = (int32_t)S, s.max_blocks_per_seq = (int32_t)table.size(1), s.num_rows = whole32(a[9]);
        s.d_block_table = ints(1, 0, "block tables are int32");
        s.d_block_refs = ints(2, l.num_blocks, "block counts are int32 [num_blocks]");
        s.d_seq_lens = ints(3, S, "lengths are int32 [num_seqs]");
        s.d_new_lens = ints(4, S, "lengths are int32 [num_seqs]");
        s.d_parents = ints(5, S, "parents are int32 [num_seqs]");
        s.d_shared_lens = ints(6, S, "shared lengths are int32 [num_seqs]");
        s.d_lens_out = ints(7, S, "lengths are int32 [num_seqs]");
        s.d_q_starts = ints(8, S + 1, "row starts are int32 [num_seqs + 1]");
        s.d_first_positions = ints(10, S, "first positions are int32 [num_seqs]");
        s.d_positions = ints(11, s.num_rows, "positions are int32 [num_rows]");
        s.d_slots = a[12] == Py_None ? nullptr : (int64_t*)dense(a[12], at::kLong, s.num_rows, dev, "slots are int64 [num_rows]");
        s.d_pairs = ints(13, 0, "pairs are int32 [pairs, 2]");
        if (s.d_pairs) {
            const at::Tensor& t = tensor(a[13]);
            if (t.dim() != 2 || t.size(1) != 2 || t.size(0) > INT32_MAX) throw Refused{"pairs are int32 [pairs, 2]"};
            s.pairs_cap = (int32_t)t.size(0);
        }
        s.d_num_pairs = ints(14, 1, "the number of pairs is int32");
        s.d_free_count = ints(15, 1, "the free count is int32");
        void* status = dense(a[16], at::kInt, 1, dev, "status is int32");
        const On here(dev, a[17]);
        return amoeba_advance_tables(&l, &s, (int32_t*)status, here.stream);
    });
}
// (layout, pools, pairs, num_pairs, layer_begin, layer_end, status, stream)
PyObject* copy_blocks(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return answer(n, 8, [&] {
        const amoeba_layout& l = layout_of(a[0]);
        const int32_t l0 = whole32(a[4]), l1 = whole32(a[5]);
        const at::Tensor& pairs = tensor(a[2]);
        const int64_t dev = pairs.is_cuda() ? pairs.device().index() : -1;
        if (pairs.dim() != 2 || pairs.size(1) != 2 || pairs.size(0) > INT32_MAX) throw Refused{"pairs are int32 [pairs, 2]"};
        Pointers pool;
        pools(a[1], l, layer_bytes(l) * l1, false, dev, &pool);
        void* pairs_p = dense(a[2], at::kInt, 0, dev, "pairs are int32 [pairs, 2]");
        void* count = dense(a[3], at::kInt, 1, dev, "the number of pairs is int32");
        void* status = dense(a[6], at::kInt, 1, dev, "status is int32");
        const On here(dev, a[7]);
        return amoeba_copy_blocks(&l, pool, (int32_t*)pairs_p, (int32_t*)count, (int32_t)pairs.size(0), l0, l1, (int32_t*)status,
                                  here.stream);
    });
}

PyMethodDef kMethods[] = {
    {"append_kv", (PyCFunction)(void (*)())append_kv, METH_FASTCALL, nullptr},
    {"attend", (PyCFunction)(void (*)())attend, METH_FASTCALL, nullptr},
    {"accumulate_scores", (PyCFunction)(void (*)())accumulate_scores, METH_FASTCALL, nullptr},
    {"attend_shared", (PyCFunction)(void (*)())attend_shared, METH_FASTCALL, nullptr},
    {"advance_tables", (PyCFunction)(void (*)())advance_tables, METH_FASTCALL, nullptr},
    {"copy_blocks", (PyCFunction)(void (*)())copy_blocks, METH_FASTCALL, nullptr},
    {"evict_kv", (PyCFunction)(void (*)())evict_kv, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls(void) { return PyModule_Create(&kModule); }
