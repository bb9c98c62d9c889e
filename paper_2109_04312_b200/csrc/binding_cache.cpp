// The per-call path of the Python binding for rotary positions and for a paged cache: argument checks, output and
// workspace allocation, the call.  Workspaces are allocated anew for every call (stream-ordered, out of torch's pool, a
// captured graph's own pool included), so that calls and graphs that overlap share none.
#include "binding.h"
#include "overlap.h"

#include <algorithm>
#include <cstring>
#include <memory>
#include <type_traits>
#include <vector>

namespace mate_binding {
namespace {

struct Library {
    decltype(&mate_rope) rope = nullptr;
    decltype(&mate_cache_extend) extend = nullptr;
    decltype(&mate_cache_append) append = nullptr;
    decltype(&mate_cache_fork) fork = nullptr;
    decltype(&mate_cache_free) free = nullptr;
    decltype(&mate_cache_compact) compact = nullptr;
    decltype(&mate_cache_workspace_bytes) workspace_bytes = nullptr;
    decltype(&mate_cache_status) status = nullptr;
    decltype(&mate_attn_decode) decode = nullptr;
    decltype(&mate_rope_axes) rope_axes = nullptr;
    decltype(&mate_cache_append_axes) append_axes = nullptr;
    decltype(&mate_cache_groups) groups = nullptr;
    decltype(&mate_attn_decode_shared) decode_shared = nullptr;
    decltype(&mate_cache_shared_workspace_bytes) shared_workspace_bytes = nullptr;
} lib;

// A cache as the calls take it; lives in a capsule of the Python object.  It holds the tensors' memory itself: an attribute of that object may be
// set to another tensor, and the calls go on with the addresses in `c`.
struct CacheInfo {
    mate_cache_t c;
    std::vector<uint8_t> head_view;
    std::vector<c10::Storage> memory;
    at::ScalarType type;
    c10::Device device;
};
const char kCapsule[] = "mate_cache_info";

const CacheInfo &cache_info(PyObject *o) {
    void *p = PyCapsule_GetPointer(o, kCapsule);
    if (!p) throw Raised();
    return *static_cast<CacheInfo *>(p);
}
// The tensors' device while a call runs, where it is not the current one.
struct OnDevice {
    c10::cuda::OptionalCUDAGuard guard;
    c10::cuda::CUDAStream stream;
    explicit OnDevice(c10::Device d)
        : guard(d.index() != c10::cuda::current_device() ? std::optional<c10::Device>(d) : std::nullopt),
          stream(c10::cuda::getCurrentCUDAStream(d.index())) {}
};

[[noreturn]] void fail_shape(const char *name, const char *what) {
    PyErr_Format(PyExc_ValueError, "%s must be %s", name, what);
    throw Raised();
}
const at::Tensor &on_gpu(PyObject *o, const char *name, const c10::Device *device) {
    if (!THPVariable_Check(o) || !THPVariable_Unpack(o).is_cuda()) fail_shape(name, "a CUDA tensor");
    const at::Tensor &t = THPVariable_Unpack(o);
    if (device && t.device() != *device) fail_shape(name, "on the device of the others");
    return t;
}
// An int32 tensor of the given shape.
const at::Tensor &int_tensor(PyObject *o, const char *name, c10::IntArrayRef shape) {
    if (!THPVariable_Check(o)) fail_shape(name, "a contiguous int32 CUDA tensor");
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.scalar_type() != at::kInt || t.sizes() != shape) {
        PyErr_Format(PyExc_ValueError, "%s must be an int32 tensor with %lld elements in %d dimension(s)", name,
                     (long long)c10::multiply_integers(shape), (int)shape.size());
        throw Raised();
    }
    return t;
}
// The same, contiguous and on the GPU; null for None where that is allowed.
int32_t *ints(PyObject *o, const char *name, c10::IntArrayRef shape, const c10::Device &device, bool may_be_none) {
    if (o == Py_None && may_be_none) return nullptr;
    const at::Tensor &t = int_tensor(o, name, shape);
    if (!t.is_cuda() || !t.is_contiguous() || t.device() != device) fail_shape(name, "a contiguous CUDA tensor on the device of the others");
    return t.data_ptr<int32_t>();
}
// Rows of contiguous elements.
void rows(const at::Tensor &t, const char *name) {
    if (t.dim() < 1 || (t.size(-1) > 1 && t.stride(-1) != 1)) fail_shape(name, "contiguous in its last dimension");
}
// No element twice (of a tensor that is written).
bool distinct(const at::Tensor &t) {
    std::vector<std::pair<int64_t, int64_t>> dims;  // stride, size
    for (int64_t i = 0; i < t.dim(); ++i)
        if (t.size(i) > 1) dims.emplace_back(t.stride(i), t.size(i));
    std::sort(dims.begin(), dims.end());
    int64_t reach = 1;
    for (const auto &[stride, size] : dims) {
        if (stride < reach) return false;
        reach = stride * (size - 1) + reach;
    }
    return true;
}
Extent extent(const at::Tensor &t) {
    Extent e = {reinterpret_cast<int64_t>(t.data_ptr()), (int64_t)t.element_size(), {}};
    for (int64_t i = 0; i < t.dim(); ++i) e.dims.emplace_back(t.stride(i) * (int64_t)t.element_size(), t.size(i));
    return e;
}
bool overlap(const at::Tensor &a, const at::Tensor &b) {
    const auto end = [](const at::Tensor &t) {
        int64_t last = 0;
        for (int64_t i = 0; i < t.dim(); ++i) last += t.stride(i) * (t.size(i) - 1);
        return reinterpret_cast<int64_t>(t.data_ptr()) + (last + 1) * (int64_t)t.element_size();
    };
    const int64_t at_a = reinterpret_cast<int64_t>(a.data_ptr()), at_b = reinterpret_cast<int64_t>(b.data_ptr());
    if (end(a) <= at_b || end(b) <= at_a) return false;  // (as most of them: no lists are made)
    return overlap(extent(a), extent(b));
}
// The same elements in the same places.
bool same_place(const at::Tensor &a, const at::Tensor &b) {
    if (a.data_ptr() != b.data_ptr() || a.scalar_type() != b.scalar_type() || a.sizes() != b.sizes()) return false;
    for (int64_t i = 0; i < a.dim(); ++i)
        if (a.size(i) > 1 && a.stride(i) != b.stride(i)) return false;
    return true;
}
int as_int(int64_t x, const char *name) {
    if (x < 0 || x > INT32_MAX) fail_shape(name, "between 0 and 2^31 - 1, and its sizes too");
    return (int)x;
}
double number(PyObject *o) {
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) throw Raised();
    return x;
}
int64_t whole(PyObject *o) {
    const long long x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) throw Raised();
    return x;
}
bool truth(PyObject *o) {
    const int x = PyObject_IsTrue(o);
    if (x < 0) throw Raised();
    return x == 1;
}
PyObject *given_or(PyObject *given, const at::Tensor &t) { return given != Py_None ? Py_NewRef(given) : THPVariable_Wrap(t); }

// Queries or keys of a rotation: [B, H, N, d] or, packed, [H, T, d].
struct Turned {
    at::Tensor x, y;
    mate_rope_tensor_t t;
};
Turned turned(PyObject *x, PyObject *y, const char *name, const char *out_name, const at::Tensor *like) {
    Turned r;
    r.x = on_gpu(x, name, nullptr);
    const at::Tensor &t = r.x;
    if (t.dim() != 3 && t.dim() != 4) fail_shape(name, "[B, H, N, d] or [H, T, d]");
    rows(t, name);
    const int o = (int)t.dim() - 4;  // -1: no batch dimension
    if (like) {
        const at::Tensor &q = *like;
        if (t.dim() != q.dim() || t.size(-1) != q.size(-1) || t.size(-2) != q.size(-2) || (o == 0 && t.size(0) != q.size(0)) ||
            t.scalar_type() != q.scalar_type() || t.device() != q.device())
            fail_shape(name, "like Q but for its number of heads");
    }
    if (y != Py_None) {
        r.y = on_gpu(y, out_name, nullptr);
        if (r.y.sizes() != t.sizes() || r.y.scalar_type() != t.scalar_type() || r.y.device() != t.device())
            fail_shape(out_name, "like what is rotated");
        rows(r.y, out_name);
        if (!distinct(r.y)) fail_shape(out_name, "a tensor without elements that share their memory");
    }
    r.t.heads = as_int(t.size(1 + o), name);
    r.t.x = t.data_ptr();
    // (the stride of a dimension of one is nobody's business: it need not fit the alignment)
    for (int i = 0; i < 3; ++i) r.t.x_stride[i] = i + o < 0 || t.size(i + o) <= 1 ? 0 : t.stride(i + o);
    return r;
}
void set_out(Turned &r) {
    if (!r.y.defined()) r.y = empty(r.x.sizes(), r.x.scalar_type(), r.x.device());
    const int o = (int)r.y.dim() - 4;
    r.t.y = r.y.data_ptr();
    for (int i = 0; i < 3; ++i) r.t.y_stride[i] = i + o < 0 || r.y.size(i + o) <= 1 ? 0 : r.y.stride(i + o);
}
// Radians per position of every pair; returns the rotated part of a row.
int frequencies(PyObject *o, int64_t d, const c10::Device &device, const double **at) {
    const at::Tensor &f = on_gpu(o, "freqs", &device);
    if (f.scalar_type() != at::kDouble || f.dim() != 1 || !f.is_contiguous()) fail_shape("freqs", "a contiguous float64 tensor [rot / 2]");
    if (2 * f.size(0) > d) fail_shape("freqs", "at most d / 2 numbers");
    static const double none = 0.;  // (an empty tensor has no address; the library takes a null one for no rotation, and then no queries)
    *at = f.size(0) ? f.data_ptr<double>() : &none;
    return (int)(2 * f.size(0));
}

// Positions of several axes, [A, ...], and the axis of every pair, as bytes.
struct Axes {
    const uint8_t *of_pair;
    int n;
    Axes(PyObject *axes, PyObject *positions, int rot) {
        if (!THPVariable_Check(positions) || THPVariable_Unpack(positions).dim() < 1) fail_shape("positions", "an int32 CUDA tensor, one row for each axis");
        n = as_int(THPVariable_Unpack(positions).size(0), "positions");
        if (!PyBytes_Check(axes) || PyBytes_GET_SIZE(axes) != rot / 2) fail_shape("axes", "one number for each frequency");
        of_pair = reinterpret_cast<const uint8_t *>(PyBytes_AS_STRING(axes));
    }
};

// rope(Q, K or None, positions, freqs, interleaved, mscale, backward, out or None, out_k or None) -> Q' or (Q', K')
// rope_axes(the same, axes)
PyObject *rope_of(PyObject *const *a, Py_ssize_t n, bool several) {
    return guarded([&]() -> PyObject * {
        if (n != 9 + several) fail(PyExc_TypeError, several ? "rope_axes takes 10 arguments" : "rope takes 9 arguments");
        Turned t[2];
        t[0] = turned(a[0], a[7], "Q", "out", nullptr);
        const bool two = a[1] != Py_None;
        if (two) t[1] = turned(a[1], a[8], "K", "out", &t[0].x);
        // An output that is given is its own input, or apart from all that is read; two of them are apart.
        for (int i = 0; i < 1 + two; ++i)
            for (int j = 0; t[i].y.defined() && j < 1 + two; ++j)
                if (i == j ? !same_place(t[i].y, t[i].x) && overlap(t[i].y, t[i].x)
                           : overlap(t[i].y, t[j].x) || (t[j].y.defined() && overlap(t[i].y, t[j].y)))
                    fail_shape("out", "the inputs themselves, or without memory in common with them, and with one another");
        const at::Tensor &Q = t[0].x;
        const c10::Device device = Q.device();
        const int dt = dtype_code(Q);
        const int64_t d = Q.size(-1), N = Q.size(-2), B = Q.dim() == 4 ? Q.size(0) : 1;
        const double *f = nullptr;
        const int rot = frequencies(a[3], d, device, &f);
        const std::optional<Axes> axes = several ? std::optional<Axes>(Axes(a[9], a[2], rot)) : std::nullopt;
        const bool one_row = THPVariable_Check(a[2]) && THPVariable_Unpack(a[2]).dim() == 1 + several;
        const int64_t all[3] = {several ? axes->n : 1, B, N}, row[2] = {all[0], N};
        const int32_t *pos = ints(a[2], "positions", one_row ? c10::IntArrayRef(row + !several, 1 + several) : c10::IntArrayRef(all + !several, 2 + several),
                                  device, false);
        const unsigned flags = (truth(a[4]) ? MATE_ROPE_INTERLEAVED : 0) | (truth(a[6]) ? MATE_ROPE_BACKWARD : 0);
        const float mscale = (float)number(a[5]);
        const int b = as_int(B, "Q"), nn = as_int(N, "Q"), dd = as_int(d, "Q");
        const OnDevice on(device);
        int status = MATE_OK;
        {
            const NoGil no_gil;
            for (int i = 0; i < 1 + two; ++i) set_out(t[i]);
            // (a tensor without elements has no address)
            mate_rope_tensor_t ts[2];
            int m = 0;
            for (int i = 0; i < 1 + two; ++i)
                if (t[i].x.numel()) ts[m++] = t[i].t;
            if (m && !several) status = lib.rope(ts, m, b, nn, dd, dt, pos, one_row ? 0 : N, f, rot, mscale, flags, on.stream.stream());
            if (m && several)
                status = lib.rope_axes(ts, m, b, nn, dd, dt, pos, one_row ? N : B * N, one_row ? 0 : N, axes->of_pair, axes->n, f, rot, mscale, flags,
                                       on.stream.stream());
        }
        check(status, several ? "mate_rope_axes" : "mate_rope");
        PyObject *q = given_or(a[7], t[0].y);
        if (!two || !q) return q;
        PyObject *k = given_or(a[8], t[1].y), *r = k ? PyTuple_Pack(2, q, k) : nullptr;
        Py_DECREF(q);
        Py_XDECREF(k);
        return r;
    });
}

PyObject *rope(PyObject *, PyObject *const *a, Py_ssize_t n) { return rope_of(a, n, false); }
PyObject *rope_axes(PyObject *, PyObject *const *a, Py_ssize_t n) { return rope_of(a, n, true); }

// cache_info(k, v, row_ids, col_ids, table, lens, prefix, refs, status, head_view bytes) -> capsule
PyObject *new_cache(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        if (n != 10) fail(PyExc_TypeError, "cache_info takes 10 arguments");
        if (!THPVariable_Check(a[0]) || !THPVariable_Check(a[1])) fail_shape("k and v", "CUDA tensors");
        const at::Tensor &k = THPVariable_Unpack(a[0]), &v = THPVariable_Unpack(a[1]);
        if (k.dim() != 5 || v.sizes() != k.sizes() || v.scalar_type() != k.scalar_type())
            fail_shape("k and v", "of one type and shape, [layers, pages, kv_heads, page_size, d]");
        const int dt = dtype_code(k);
        rows(k, "k"), rows(v, "v");
        if (k.strides() != v.strides() || !distinct(k) || overlap(k, v))
            fail_shape("k and v", "laid out alike, without elements that share their memory");
        if (!THPVariable_Check(a[4]) || THPVariable_Unpack(a[4]).dim() != 2) fail_shape("table", "an int32 CUDA tensor [seqs, width]");
        const at::Tensor &table = THPVariable_Unpack(a[4]);
        if (!PyBytes_Check(a[9])) fail_shape("head_view", "bytes");
        const int64_t pages = k.size(1), page_size = k.size(3), seqs = table.size(0), width = table.size(1);
        const c10::Device device = k.device();
        auto info = std::make_unique<CacheInfo>(CacheInfo{{}, {}, {}, k.scalar_type(), device});
        mate_cache_t &c = info->c;
        struct {
            int32_t **to;
            const char *name;
            std::vector<int64_t> shape;
        } arrays[] = {{&c.row_ids, "row_ids", {pages, page_size}}, {&c.col_ids, "col_ids", {pages, page_size}}, {&c.table, "table", {seqs, width}},
                      {&c.lens, "lens", {seqs}}, {&c.prefix, "prefix", {seqs}}, {&c.refs, "refs", {pages}}, {&c.status, "status", {1}}};
        for (int i = 0; i < 7; ++i) int_tensor(a[2 + i], arrays[i].name, arrays[i].shape);
        for (int i = 0; i < 7; ++i) *arrays[i].to = ints(a[2 + i], arrays[i].name, arrays[i].shape, device, false);
        if (!k.is_cuda() || v.device() != device) fail_shape("k and v", "CUDA tensors on one device");
        const uint8_t *view = reinterpret_cast<const uint8_t *>(PyBytes_AS_STRING(a[9]));
        info->head_view.assign(view, view + PyBytes_GET_SIZE(a[9]));
        for (int i = 0; i < 9; ++i) info->memory.push_back(THPVariable_Unpack(a[i]).storage());
        c.k = k.data_ptr(), c.v = v.data_ptr();
        c.head_view = info->head_view.data();
        // (a stride that nothing is multiplied by need not fit the alignment)
        const auto stride = [&](int i) { return k.size(i) > 1 ? k.stride(i) : 0; };
        c.layer_stride = stride(0), c.page_stride = stride(1), c.head_stride = stride(2), c.slot_stride = stride(3);
        c.layers = as_int(k.size(0), "k"), c.pages = as_int(pages, "k"), c.kv_heads = as_int(k.size(2), "k");
        c.page_size = as_int(page_size, "k"), c.d = as_int(k.size(4), "k");
        c.seqs = as_int(seqs, "table"), c.width = as_int(width, "table");
        c.heads = as_int((int64_t)info->head_view.size(), "head_view"), c.dtype = dt, c.device = device.index();
        check(lib.workspace_bytes(&c, 0, nullptr, nullptr, nullptr), "Cache");
        return PyCapsule_New(info.release(), kCapsule,
                             [](PyObject *o) { delete static_cast<CacheInfo *>(PyCapsule_GetPointer(o, kCapsule)); });
    });
}

// Entries of a list of sequences, for which None stands for all of them in order.
int entries(PyObject *list, PyObject *other, const char *name) {
    PyObject *o = list != Py_None ? list : other;
    if (!THPVariable_Check(o) || THPVariable_Unpack(o).dim() != 1) fail_shape(name, "an int32 CUDA tensor [n]");
    return as_int(THPVariable_Unpack(o).size(0), name);
}

// cache_extend(info, seqs or None, counts, granted or None) -> granted
PyObject *cache_extend(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        if (n != 4) fail(PyExc_TypeError, "cache_extend takes 4 arguments");
        const CacheInfo &ci = cache_info(a[0]);
        const int m = entries(a[1], a[2], "seqs");
        const int32_t *seqs = ints(a[1], "seqs", {m}, ci.device, true), *counts = ints(a[2], "counts", {m}, ci.device, false);
        int32_t *granted = ints(a[3], "granted", {m}, ci.device, true);
        at::Tensor out;
        const OnDevice on(ci.device);
        int status;
        {
            const NoGil no_gil;
            if (!granted) out = empty({m}, at::kInt, ci.device), granted = out.data_ptr<int32_t>();
            status = lib.extend(&ci.c, seqs, counts, m, granted, on.stream.stream());
        }
        check(status, "mate_cache_extend");
        return given_or(a[3], out);
    });
}

// cache_append(info, layer, K, V, seqs, counts, row_ids, col_ids, positions, freqs, interleaved, mscale, Q, out) -> rotated Q or None
// cache_append_axes(the same, axes)
PyObject *append_of(PyObject *const *a, Py_ssize_t n, bool several) {
    return guarded([&]() -> PyObject * {
        if (n != 14 + several) fail(PyExc_TypeError, several ? "cache_append_axes takes 15 arguments" : "cache_append takes 14 arguments");
        const CacheInfo &ci = cache_info(a[0]);
        const int layer = as_int(whole(a[1]), "layer");
        const at::Tensor &K = on_gpu(a[2], "K", &ci.device), &V = on_gpu(a[3], "V", &ci.device);
        int64_t ks[3], vs[3];
        for (const auto &[t, strides] : {std::pair(&K, ks), std::pair(&V, vs)}) {  // (K and V may be one tensor)
            if (t->dim() != 4 || t->size(1) != ci.c.kv_heads || t->size(3) != ci.c.d || t->sizes() != K.sizes() || t->scalar_type() != ci.type)
                fail_shape("K and V", "[B, kv_heads, N, d] of the cache's type");
            rows(*t, "K and V");
            for (int i = 0; i < 3; ++i) strides[i] = t->size(i) > 1 ? t->stride(i) : 0;
        }
        const int64_t B = K.size(0), N = K.size(2);
        const int32_t *seqs = ints(a[4], "seqs", {B}, ci.device, true), *counts = ints(a[5], "counts", {B}, ci.device, true);
        const int32_t *row = ints(a[6], "row_ids", {B, N}, ci.device, true), *col = ints(a[7], "col_ids", {B, N}, ci.device, true);
        const double *f = nullptr;
        const int rot = a[9] == Py_None && !several ? 0 : frequencies(a[9], ci.c.d, ci.device, &f);
        const std::optional<Axes> axes = several ? std::optional<Axes>(Axes(a[14], a[8], rot)) : std::nullopt;
        const int64_t all[3] = {several ? axes->n : 1, B, N};
        const int32_t *pos = ints(a[8], "positions", c10::IntArrayRef(all + !several, 2 + several), ci.device, !several);
        const unsigned flags = truth(a[10]) ? MATE_ROPE_INTERLEAVED : 0;
        const float mscale = (float)number(a[11]);
        const bool with_q = a[12] != Py_None;
        if (!with_q && a[13] != Py_None) fail(PyExc_ValueError, "out must be None where no Q is given");
        Turned q = {};
        if (with_q) {
            q = turned(a[12], a[13], "Q", "out", nullptr);
            if (q.x.dim() != 4 || q.x.size(0) != B || q.x.size(1) != ci.c.heads || q.x.size(2) != N || q.x.size(3) != ci.c.d ||
                q.x.scalar_type() != ci.type || q.x.device() != ci.device)
                fail_shape("Q", "[B, heads, N, d] of the cache's type");
            if (q.y.defined() && ((!same_place(q.y, q.x) && overlap(q.y, q.x)) || overlap(q.y, K) || overlap(q.y, V)))
                fail_shape("out", "Q itself, or without memory in common with Q, K and V");
        }
        const int b = as_int(B, "K"), nn = as_int(N, "K");
        const OnDevice on(ci.device);
        int status = MATE_OK;
        {
            const NoGil no_gil;
            if (with_q) set_out(q);
            const void *qx = with_q ? q.t.x : nullptr;
            void *qy = with_q ? q.t.y : nullptr;
            if (b > 0 && nn > 0 && !several)
                status = lib.append(&ci.c, layer, K.data_ptr(), V.data_ptr(), ks, vs, b, nn, seqs, counts, row, col, pos, f, rot, mscale, flags,
                                    qx, q.t.x_stride, qy, q.t.y_stride, on.stream.stream());
            if (b > 0 && nn > 0 && several)
                status = lib.append_axes(&ci.c, layer, K.data_ptr(), V.data_ptr(), ks, vs, b, nn, seqs, counts, row, col, pos, axes->of_pair, axes->n, f,
                                         rot, mscale, flags, qx, q.t.x_stride, qy, q.t.y_stride, on.stream.stream());
        }
        check(status, several ? "mate_cache_append_axes" : "mate_cache_append");
        if (!with_q) Py_RETURN_NONE;
        return given_or(a[13], q.y);
    });
}

PyObject *cache_append(PyObject *, PyObject *const *a, Py_ssize_t n) { return append_of(a, n, false); }
PyObject *cache_append_axes(PyObject *, PyObject *const *a, Py_ssize_t n) { return append_of(a, n, true); }

// Workspace of one call.
struct Scratch {
    at::Tensor t;
    void *ptr = nullptr;
    size_t bytes = 0;
    Scratch(size_t need, const c10::Device &device) {
        if (!need) return;
        t = empty({(int64_t)need}, at::kByte, device);
        ptr = t.data_ptr(), bytes = need;
    }
};

// cache_fork(info, parents, children)
PyObject *cache_fork(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        if (n != 3) fail(PyExc_TypeError, "cache_fork takes 3 arguments");
        const CacheInfo &ci = cache_info(a[0]);
        const int m = entries(a[1], a[2], "parents");
        const int32_t *parents = ints(a[1], "parents", {m}, ci.device, false), *children = ints(a[2], "children", {m}, ci.device, false);
        const OnDevice on(ci.device);
        size_t need = 0;
        check(lib.workspace_bytes(&ci.c, m, &need, nullptr, nullptr), "mate_cache_fork");
        int status;
        {
            const NoGil no_gil;
            const Scratch ws(need, ci.device);
            status = lib.fork(&ci.c, parents, children, m, ws.ptr, ws.bytes, on.stream.stream());
        }
        check(status, "mate_cache_fork");
        Py_RETURN_NONE;
    });
}

// cache_free(info, seqs or None)
PyObject *cache_free(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        if (n != 2) fail(PyExc_TypeError, "cache_free takes 2 arguments");
        const CacheInfo &ci = cache_info(a[0]);
        const int m = a[1] == Py_None ? ci.c.seqs : entries(a[1], a[1], "seqs");
        const int32_t *seqs = ints(a[1], "seqs", {m}, ci.device, true);
        const OnDevice on(ci.device);
        int status;
        {
            const NoGil no_gil;
            status = lib.free(&ci.c, seqs, m, on.stream.stream());
        }
        check(status, "mate_cache_free");
        Py_RETURN_NONE;
    });
}

// cache_compact(info, n_live or None) -> n_live
PyObject *cache_compact(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        if (n != 2) fail(PyExc_TypeError, "cache_compact takes 2 arguments");
        const CacheInfo &ci = cache_info(a[0]);
        int32_t *live = ints(a[1], "n_live", {}, ci.device, true);
        at::Tensor out;
        const OnDevice on(ci.device);
        size_t need = 0;
        check(lib.workspace_bytes(&ci.c, 0, nullptr, &need, nullptr), "mate_cache_compact");
        int status;
        {
            const NoGil no_gil;
            if (!live) out = empty({}, at::kInt, ci.device), live = out.data_ptr<int32_t>();
            const Scratch ws(need, ci.device);
            status = lib.compact(&ci.c, live, ws.ptr, ws.bytes, on.stream.stream());
        }
        check(status, "mate_cache_compact");
        return given_or(a[1], out);
    });
}

// cache_groups(info, seqs or None, min_len, out or None) -> groups
PyObject *cache_groups(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        if (n != 4) fail(PyExc_TypeError, "cache_groups takes 4 arguments");
        const CacheInfo &ci = cache_info(a[0]);
        const int m = a[1] == Py_None ? ci.c.seqs : entries(a[1], a[1], "seqs"), min_len = as_int(whole(a[2]), "min_len");
        const int32_t *seqs = ints(a[1], "seqs", {m}, ci.device, true);
        int32_t *groups = ints(a[3], "out", {3, m}, ci.device, true);
        if (groups && seqs && overlap(THPVariable_Unpack(a[3]), THPVariable_Unpack(a[1]))) fail_shape("out", "without memory in common with seqs");
        at::Tensor out;
        const OnDevice on(ci.device);
        int status;
        {
            const NoGil no_gil;
            if (!groups) out = empty({3, m}, at::kInt, ci.device), groups = out.data_ptr<int32_t>();
            status = lib.groups(&ci.c, seqs, m, min_len, groups, on.stream.stream());
        }
        check(status, "mate_cache_groups");
        return given_or(a[3], out);
    });
}

// cache_status(info)
PyObject *cache_status(PyObject *, PyObject *o) {
    return guarded([&]() -> PyObject * {
        const CacheInfo &ci = cache_info(o);
        const OnDevice on(ci.device);
        int status;
        {
            const NoGil no_gil;
            status = lib.status(&ci.c, on.stream.stream());
        }
        check(status, "mate_cache_status");
        Py_RETURN_NONE;
    });
}

// attn_decode(info, layer, Q, seqs, row_ids, col_ids, scale, max_len, out, lse) -> (O, LSE)
// attn_decode_shared(the same, groups, always)
PyObject *decode_of(PyObject *const *a, Py_ssize_t n, bool shared) {
    return guarded([&]() -> PyObject * {
        if (n != (shared ? 12 : 10)) fail(PyExc_TypeError, shared ? "attn_decode_shared takes 12 arguments" : "attn_decode takes 10 arguments");
        const CacheInfo &ci = cache_info(a[0]);
        const int layer = as_int(whole(a[1]), "layer");
        const at::Tensor &Q = on_gpu(a[2], "Q", &ci.device);
        if (Q.dim() != 3 || Q.size(1) != ci.c.heads || Q.size(2) != ci.c.d || Q.scalar_type() != ci.type)
            fail_shape("Q", "[B, heads, d] of the cache's type");
        rows(Q, "Q");
        const int64_t B = Q.size(0);
        const int32_t *seqs = ints(a[3], "seqs", {B}, ci.device, true);
        const int32_t *row = ints(a[4], "row_ids", {B}, ci.device, false), *col = ints(a[5], "col_ids", {B}, ci.device, false);
        const int32_t *groups = shared ? ints(a[10], "groups", {3, B}, ci.device, false) : nullptr;
        const float scale = scale_of(a[6], ci.c.d);
        const int max_len = a[7] == Py_None ? 0 : as_int(whole(a[7]), "max_len");
        if (a[7] != Py_None && max_len == 0) fail_shape("max_len", "positive");
        const int always = shared ? PyObject_IsTrue(a[11]) : 0;
        if (always < 0) throw Raised();
        at::Tensor O, LSE;
        if (a[8] != Py_None) {
            O = on_gpu(a[8], "O", &ci.device);
            if (O.sizes() != Q.sizes() || O.scalar_type() != ci.type || !O.is_contiguous()) fail_shape("O", "a contiguous tensor like Q");
        }
        if (a[9] != Py_None) {
            LSE = on_gpu(a[9], "LSE", &ci.device);
            if (LSE.sizes() != Q.sizes().slice(0, 2) || LSE.scalar_type() != at::kFloat || !LSE.is_contiguous())
                fail_shape("LSE", "a contiguous float32 tensor [B, heads]");
        }
        if (O.defined() && !same_place(O, Q) && overlap(O, Q)) fail_shape("O", "Q itself, or without memory in common with it");
        if (LSE.defined() && (overlap(LSE, Q) || (O.defined() && overlap(LSE, O)))) fail_shape("LSE", "without memory in common with Q and O");
        const int64_t qs[2] = {B > 1 ? Q.stride(0) : 0, ci.c.heads > 1 ? Q.stride(1) : 0};
        const int b = as_int(B, "Q");
        const OnDevice on(ci.device);
        size_t need = 0;
        const char *name = shared ? "mate_attn_decode_shared" : "mate_attn_decode";
        check(shared ? lib.shared_workspace_bytes(&ci.c, b, &need) : lib.workspace_bytes(&ci.c, b, nullptr, nullptr, &need), name);
        int status;
        {
            const NoGil no_gil;
            if (!O.defined()) O = empty(Q.sizes(), ci.type, ci.device);
            if (!LSE.defined()) LSE = empty(Q.sizes().slice(0, 2), at::kFloat, ci.device);
            const Scratch ws(b ? need : 0, ci.device);
            status = shared ? lib.decode_shared(&ci.c, layer, Q.data_ptr(), qs, b, seqs, row, col, groups, scale, max_len,
                                                always ? MATE_SHARED_ALWAYS : 0, O.data_ptr(), LSE.data_ptr<float>(), ws.ptr, ws.bytes, on.stream.stream())
                            : lib.decode(&ci.c, layer, Q.data_ptr(), qs, b, seqs, row, col, scale, max_len, O.data_ptr(), LSE.data_ptr<float>(),
                                         ws.ptr, ws.bytes, on.stream.stream());
        }
        check(status, name);
        PyObject *po = given_or(a[8], O), *pl = given_or(a[9], LSE), *r = po && pl ? PyTuple_Pack(2, po, pl) : nullptr;
        Py_XDECREF(po);
        Py_XDECREF(pl);
        return r;
    });
}

PyObject *attn_decode(PyObject *, PyObject *const *a, Py_ssize_t n) { return decode_of(a, n, false); }
PyObject *attn_decode_shared(PyObject *, PyObject *const *a, Py_ssize_t n) { return decode_of(a, n, true); }

// bind_cache(addresses of the library's entry points, in the order of Library)
PyObject *bind_cache(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded([&]() -> PyObject * {
        void *p[sizeof(Library) / sizeof(void *)];
        if (n != (Py_ssize_t)(sizeof p / sizeof *p)) fail(PyExc_TypeError, "bind_cache takes an address for each entry point");
        for (Py_ssize_t i = 0; i < n; ++i) {
            p[i] = PyLong_AsVoidPtr(a[i]);
            if (PyErr_Occurred()) throw Raised();
        }
        static_assert(sizeof(Library) == sizeof p && std::is_trivially_copyable_v<Library>, "addresses and nothing else");
        std::memcpy(&lib, p, sizeof p);
        Py_RETURN_NONE;
    });
}

}  // namespace

PyMethodDef cache_methods[] = {{"rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(rope)), METH_FASTCALL, nullptr},
                               {"cache_info", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(new_cache)), METH_FASTCALL, nullptr},
                               {"cache_extend", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(cache_extend)), METH_FASTCALL, nullptr},
                               {"cache_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(cache_append)), METH_FASTCALL, nullptr},
                               {"cache_fork", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(cache_fork)), METH_FASTCALL, nullptr},
                               {"cache_free", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(cache_free)), METH_FASTCALL, nullptr},
                               {"cache_compact", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(cache_compact)), METH_FASTCALL, nullptr},
                               {"cache_groups", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(cache_groups)), METH_FASTCALL, nullptr},
                               {"cache_status", cache_status, METH_O, nullptr},
                               {"attn_decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(attn_decode)), METH_FASTCALL, nullptr},
                               {"attn_decode_shared", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(attn_decode_shared)), METH_FASTCALL, nullptr},
                               {"rope_axes", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(rope_axes)), METH_FASTCALL, nullptr},
                               {"cache_append_axes", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(cache_append_axes)), METH_FASTCALL, nullptr},
                               {"bind_cache", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(bind_cache)), METH_FASTCALL, nullptr},
                               {nullptr, nullptr, 0, nullptr}};

}  // namespace mate_binding
