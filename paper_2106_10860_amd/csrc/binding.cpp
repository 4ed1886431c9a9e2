// Argument marshalling of the Python calls that a program makes over and over, in native code.
//
// A call on few rows is shorter on the device (4 to 6 us) than its way through the Python binding was (3.6 us of checks and
// ctypes, 1.5 for the result, 2.5 for the launch), so that the host bound it: 1000 rows of 320 floats, C = 16, M = 128 took 8.0 us a
// call whatever the kernel did.  These functions take the tensors apart through torch's C++ interface and call the same entry
// points of libmaddness.  They look at the usual arguments only - plain tensors on the device, of the type and shape the
// call wants - and return NotImplemented for anything else, after which the Python code does the call, or raises.
// A status other than MADDNESS_OK comes back as a number.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/core/Allocator.h>
#include <c10/core/GradMode.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdio>
#include <cstring>
#include <vector>

#include "maddness.h"

namespace {

struct NotUsual {};

PyObject *s_split_dims, *s_thresholds, *s_prototypes, *s_C, *s_D, *s_cuda_stream, *s_q, *s_scale, *s_tile;
PyObject *get_stream, *get_device;     // torch._C._cuda_getCurrentRawStream, _cuda_getDevice
PyObject *int_status(int rc) { return PyLong_FromLong(rc); }

// A new reference that ends with the scope.
struct Ref {
    PyObject *p;
    explicit Ref(PyObject *o) : p(o)
    {
        if (!p) {
            PyErr_Clear();
            throw NotUsual();
        }
    }
    ~Ref() { Py_DECREF(p); }
    Ref(const Ref &) = delete;
};

const at::Tensor &tensor(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) throw NotUsual();
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.layout() != at::kStrided) throw NotUsual();
    return t;
}

template <typename T>
T *pointer(PyObject *o, at::ScalarType type)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o);
    if (t.scalar_type() != type) throw NotUsual();
    return static_cast<T *>(t.data_ptr());
}

uint16_t *sums(PyObject *o)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o);
    if (t.scalar_type() != at::kShort && t.scalar_type() != at::kUInt16) throw NotUsual();
    return static_cast<uint16_t *>(t.data_ptr());
}

struct Rows {
    int64_t rows, cols, ld;
};

// rows, columns and row stride of a matrix whose rows are contiguous
Rows rows_of(const at::Tensor &t)
{
    if (t.dim() != 2) throw NotUsual();
    const int64_t r = t.size(0), c = t.size(1), s = t.stride(0);
    if (c > 1 && t.stride(1) != 1) throw NotUsual();
    return {r, c, r > 1 ? s : std::max(c, s)};
}

int64_t whole(PyObject *o)
{
    if (!PyLong_CheckExact(o)) throw NotUsual();
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw NotUsual();
    }
    return v;
}

void *stream_of(PyObject *stream)
{
    if (stream != Py_None) {
        Ref raw(PyObject_GetAttr(stream, s_cuda_stream));
        return reinterpret_cast<void *>(whole(raw.p));
    }
    Ref device(PyObject_CallNoArgs(get_device));
    Ref raw(PyObject_CallOneArg(get_stream, device.p));
    return reinterpret_cast<void *>(whole(raw.p));
}

// The trees (and D where the parameters know it) of a Params object.
maddness_params params_of(PyObject *o, int64_t D)
{
    maddness_params p{};
    Ref C(PyObject_GetAttr(o, s_C)), split(PyObject_GetAttr(o, s_split_dims)), th(PyObject_GetAttr(o, s_thresholds)),
        proto(PyObject_GetAttr(o, s_prototypes));
    const int64_t c = whole(C.p);
    if (D > INT32_MAX || c > INT32_MAX || c < INT32_MIN) throw NotUsual();
    p.D = (int32_t)D;
    p.C = (int32_t)c;
    p.split_dims = pointer<int32_t>(split.p, at::kInt);
    p.thresholds = pointer<float>(th.p, at::kFloat);
    p.prototypes = pointer<float>(proto.p, at::kFloat);
    return p;
}

int64_t own_D(PyObject *o)
{
    Ref d(PyObject_GetAttr(o, s_D));
    return d.p == Py_None ? -1 : whole(d.p);
}

int32_t narrow(int64_t v)
{
    if (v > INT32_MAX || v < INT32_MIN) throw NotUsual();
    return (int32_t)v;
}

bool truth(PyObject *o)
{
    if (o != Py_True && o != Py_False) throw NotUsual();
    return o == Py_True;
}

int type_of(const at::Tensor &t)
{
    switch (t.scalar_type()) {
    case at::kFloat: return MADDNESS_F32;
    case at::kHalf: return MADDNESS_F16;
    case at::kBFloat16: return MADDNESS_BF16;
    case at::kByte: return MADDNESS_U8;
    default: throw NotUsual();
    }
}

int64_t columns_of_tables(PyObject *luts)
{
    const at::Tensor &t = tensor(luts);
    if (t.dim() != 3) throw NotUsual();
    return t.size(2);
}

// Runs f; whatever is not usual, or goes wrong before the library is called, is left to the Python code.
template <typename F>
PyObject *usual(F f)
{
    try {
        return f();
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NOTIMPLEMENTED;
    }
}

// (kind, col_major, params, A, luts, scale, offset, out, acc, codes, want_out, stream); kind 0: fp32 rows, 1: fp32 rows and
// averages, 2: typed
PyObject *encode_scan(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 12) throw NotUsual();
        const int64_t kind = whole(a[0]);
        const bool col_major = truth(a[1]);
        const at::Tensor &A = tensor(a[3]);
        const int dtype = type_of(A);
        if (kind != 2 && dtype != MADDNESS_F32) throw NotUsual();
        const Rows ra = rows_of(A);
        const int64_t N = col_major ? ra.cols : ra.rows, D = col_major ? ra.rows : ra.cols;
        const int32_t M = narrow(columns_of_tables(a[4]));
        const maddness_params p = params_of(a[2], D);
        const void *A_p = A.data_ptr();
        const uint8_t *luts = pointer<uint8_t>(a[4], at::kByte);
        const float *scale = pointer<float>(a[5], at::kFloat), *offset = pointer<float>(a[6], at::kFloat);
        uint16_t *acc = sums(a[8]);
        uint8_t *codes = pointer<uint8_t>(a[9], at::kByte);
        void *stream = stream_of(a[11]);
        at::Tensor made;
        float *out = nullptr;
        int64_t ldo = 0;
        if (a[7] != Py_None) {
            out = pointer<float>(a[7], at::kFloat);
            ldo = rows_of(tensor(a[7])).ld;
        } else if (truth(a[10])) {
            made = at::empty({N, M}, at::TensorOptions().dtype(at::kFloat).device(A.device()));
            out = static_cast<float *>(made.data_ptr());
            ldo = rows_of(made).ld;
        }
        int rc;
        Py_BEGIN_ALLOW_THREADS
        if (kind == 2)
            rc = maddness_encode_scan_typed(&p, A_p, dtype, col_major ? MADDNESS_COL_MAJOR : MADDNESS_ROW_MAJOR, N, ra.ld, M, luts, scale,
                                            offset, out, ldo, acc, codes, stream);
        else if (kind == 1)
            rc = maddness_encode_scan_averaged(&p, static_cast<const float *>(A_p), N, ra.ld, M, luts, scale, offset, out, ldo, acc, codes,
                                               stream);
        else
            rc = maddness_encode_scan(&p, static_cast<const float *>(A_p), N, ra.ld, M, luts, scale, offset, out, ldo, acc, codes, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        if (made.defined()) return THPVariable_Wrap(std::move(made));
        Py_INCREF(a[7]);
        return a[7];
    });
}

// (kind, col_major, params, A, codes, stream); kind 0: fp32 rows, 2: typed
PyObject *encode(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 6) throw NotUsual();
        const int64_t kind = whole(a[0]);
        const bool col_major = truth(a[1]);
        const at::Tensor &A = tensor(a[3]);
        const int dtype = type_of(A);
        if (kind != 2 && dtype != MADDNESS_F32) throw NotUsual();
        const Rows ra = rows_of(A);
        const int64_t N = col_major ? ra.cols : ra.rows, D = col_major ? ra.rows : ra.cols, known = own_D(a[2]);
        if (known != -1 && known != D) throw NotUsual();
        const maddness_params p = params_of(a[2], D);
        const void *A_p = A.data_ptr();
        void *stream = stream_of(a[5]);
        at::Tensor made;
        uint8_t *codes;
        if (a[4] != Py_None) {
            codes = pointer<uint8_t>(a[4], at::kByte);
        } else {
            made = at::empty({N, ((int64_t)p.C + 1) / 2}, at::TensorOptions().dtype(at::kByte).device(A.device()));
            codes = static_cast<uint8_t *>(made.data_ptr());
        }
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = kind == 2 ? maddness_encode_typed(&p, A_p, dtype, col_major ? MADDNESS_COL_MAJOR : MADDNESS_ROW_MAJOR, N, ra.ld, codes, stream)
                       : maddness_encode(&p, static_cast<const float *>(A_p), N, ra.ld, codes, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        if (made.defined()) return THPVariable_Wrap(std::move(made));
        Py_INCREF(a[4]);
        return a[4];
    });
}

// (averaged, n_codebooks, codes, luts, scale, offset, out, acc, want_out, stream) -> out
PyObject *scan(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 10) throw NotUsual();
        const bool averaged = truth(a[0]);
        const int32_t C = narrow(whole(a[1]));
        const at::Tensor &codes = tensor(a[2]);
        if (codes.dim() < 1) throw NotUsual();
        const int64_t N = codes.size(0);
        const int32_t M = narrow(columns_of_tables(a[3]));
        const uint8_t *codes_p = pointer<uint8_t>(a[2], at::kByte), *luts = pointer<uint8_t>(a[3], at::kByte);
        const float *scale = pointer<float>(a[4], at::kFloat), *offset = pointer<float>(a[5], at::kFloat);
        uint16_t *acc = sums(a[7]);
        void *stream = stream_of(a[9]);
        at::Tensor made;
        float *out = nullptr;
        int64_t ldo = 0;
        if (a[6] != Py_None) {
            out = pointer<float>(a[6], at::kFloat);
            ldo = rows_of(tensor(a[6])).ld;
        } else if (truth(a[8])) {
            made = at::empty({N, M}, at::TensorOptions().dtype(at::kFloat).device(codes.device()));
            out = static_cast<float *>(made.data_ptr());
            ldo = rows_of(made).ld;
        }
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = averaged ? maddness_scan_averaged(C, M, codes_p, N, luts, scale, offset, out, ldo, acc, stream)
                      : maddness_scan(C, M, codes_p, N, luts, scale, offset, out, ldo, acc, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        if (made.defined()) return THPVariable_Wrap(std::move(made));
        Py_INCREF(a[6]);
        return a[6];
    });
}

// (pooled, params, B, luts, scale, offset, workspace, stream) -> (luts, scale, offset)
PyObject *build_luts(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 8) throw NotUsual();
        const bool pooled = truth(a[0]);
        const at::Tensor &B = tensor(a[2]);
        const Rows rb = rows_of(B);
        if (own_D(a[1]) != rb.rows) throw NotUsual();
        const maddness_params p = params_of(a[1], rb.rows);
        const int32_t M = narrow(rb.cols);
        const float *B_p = pointer<float>(a[2], at::kFloat);
        void *stream = stream_of(a[7]);
        const auto bytes = at::TensorOptions().dtype(at::kByte).device(B.device()), floats = bytes.dtype(at::kFloat);
        const at::Tensor luts = a[3] == Py_None ? at::empty({p.C, 16, M}, bytes) : tensor(a[3]);
        const at::Tensor scale = a[4] == Py_None ? at::empty({M}, floats) : tensor(a[4]);
        const at::Tensor offset = a[5] == Py_None ? at::empty({M}, floats) : tensor(a[5]);
        const at::Tensor work = a[6] == Py_None ? at::empty({(int64_t)maddness_build_luts_workspace(p.D, p.C, M)}, bytes) : tensor(a[6]);
        if (luts.scalar_type() != at::kByte || scale.scalar_type() != at::kFloat || offset.scalar_type() != at::kFloat ||
            work.scalar_type() != at::kByte)
            throw NotUsual();
        uint8_t *luts_p = static_cast<uint8_t *>(luts.data_ptr());
        float *scale_p = static_cast<float *>(scale.data_ptr()), *offset_p = static_cast<float *>(offset.data_ptr());
        void *work_p = work.data_ptr();
        const size_t work_bytes = (size_t)work.numel();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = (pooled ? maddness_build_luts_pooled : maddness_build_luts)(&p, B_p, M, rb.ld, luts_p, scale_p, offset_p, work_p, work_bytes,
                                                                         stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        PyObject *three[3];
        for (int k = 0; k < 3; ++k) {
            if (a[3 + k] == Py_None) {
                three[k] = THPVariable_Wrap(k == 0 ? luts : k == 1 ? scale : offset);
            } else {
                Py_INCREF(a[3 + k]);
                three[k] = a[3 + k];
            }
        }
        PyObject *tuple = PyTuple_New(3);
        for (int k = 0; k < 3; ++k) PyTuple_SET_ITEM(tuple, k, three[k]);
        return tuple;
    });
}

// ------------------------------------------------------------------------------------- 8-bit block matrices and experts

// The dtype code of a floating type.
int float_code(at::ScalarType t)
{
    if (t == at::kBFloat16) return MADDNESS_BF16;
    if (t == at::kFloat) return MADDNESS_F32;
    if (t == at::kHalf) return MADDNESS_F16;
    throw NotUsual();
}

at::ScalarType dtype_or(PyObject *o, at::ScalarType otherwise)
{
    if (o == Py_None) return otherwise;
    if (!THPDtype_Check(o)) throw NotUsual();
    return reinterpret_cast<THPDtype *>(o)->scalar_type;
}

int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// A tensor that nothing is to be recorded of: the Python code says so of one that has a gradient.
const at::Tensor &plain(PyObject *o)
{
    const at::Tensor &t = tensor(o);
    if (t.requires_grad() && c10::GradMode::is_enabled()) throw NotUsual();
    return t;
}

// A contiguous tensor of this type and these sizes.
const at::Tensor &flat(PyObject *o, at::ScalarType type, at::IntArrayRef sizes, const at::Device &device)
{
    const at::Tensor &t = plain(o);
    if (t.scalar_type() != type || t.sizes() != sizes || !t.is_contiguous() || t.device() != device) throw NotUsual();
    return t;
}

template <typename T>
T *flat_or_null(PyObject *o, at::ScalarType type, at::IntArrayRef sizes, const at::Device &device)
{
    return o == Py_None ? nullptr : static_cast<T *>(flat(o, type, sizes, device).data_ptr());
}

// A BlockMatrix: what its constructor checks, as its parts may have been replaced since.
maddness_block_matrix block_matrix(PyObject *o, const at::Device *device, int64_t *experts, at::Device *own = nullptr)
{
    Ref q_ref(PyObject_GetAttr(o, s_q)), scale_ref(PyObject_GetAttr(o, s_scale)), tile(PyObject_GetAttr(o, s_tile));
    const at::Tensor &q = tensor(q_ref.p), &scale = tensor(scale_ref.p);
    const int64_t n = q.dim();
    if (n != scale.dim() || (n != 2 && n != 3) || q.scalar_type() != at::kFloat8_e4m3fn || (device && q.device() != *device)) throw NotUsual();
    maddness_block_matrix m{};
    m.data = q.data_ptr();
    m.dtype = MADDNESS_E4M3;
    m.tile = narrow(whole(tile.p));
    m.rows = q.size(n - 2);
    m.cols = q.size(n - 1);
    if ((m.tile != 1 && m.tile != MADDNESS_BLOCK) || scale.scalar_type() != at::kByte || scale.device() != q.device() || (n == 3 && scale.size(0) != q.size(0)) ||
        scale.size(n - 2) != (m.rows + m.tile - 1) / m.tile || scale.size(n - 1) < (m.cols + MADDNESS_BLOCK - 1) / MADDNESS_BLOCK || (m.cols > 1 && q.stride(n - 1) != 1) ||
        (scale.size(n - 1) > 1 && scale.stride(n - 1) != 1))
        throw NotUsual();
    m.ld = m.rows > 1 ? q.stride(n - 2) : up(std::max(m.cols, q.stride(n - 2)), 16);
    m.scale = static_cast<const uint8_t *>(scale.data_ptr());
    m.lds = scale.size(n - 2) > 1 ? scale.stride(n - 2) : up(std::max(scale.size(n - 1), scale.stride(n - 2)), 4);
    *experts = n == 3 ? q.size(0) : -1;
    if (n == 3 && q.size(0) > 1) {
        m.stride = q.stride(0);
        m.scale_stride = scale.stride(0);
    }
    if (own) *own = q.device();
    return m;
}

struct NewBlocks {
    at::Tensor q, scale;
    int64_t ld, lds;
};

NewBlocks new_blocks(int64_t count, int64_t rows, int64_t cols, int64_t tile, const at::Device &device)
{
    NewBlocks b;
    b.ld = up(cols, 16);
    b.lds = up((cols + MADDNESS_BLOCK - 1) / MADDNESS_BLOCK, 4);
    const auto bytes = at::TensorOptions().dtype(at::kByte).device(device), e4m3 = bytes.dtype(at::kFloat8_e4m3fn);
    const int64_t exp_rows = (rows + tile - 1) / tile;
    b.q = count < 0 ? at::empty({rows, b.ld}, e4m3) : at::empty({count, rows, b.ld}, e4m3);
    b.scale = count < 0 ? at::empty({exp_rows, b.lds}, bytes) : at::empty({count, exp_rows, b.lds}, bytes);
    if (b.ld != cols) b.q = b.q.narrow(-1, 0, cols);
    return b;
}

// (x, tile, transposed, both, source, repeat, factors) -> (q, scale) or (q, scale, qt, scale_t)
PyObject *quantise_blocks(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 7) throw NotUsual();
        const at::Tensor &x = plain(a[0]);
        const int code = float_code(x.scalar_type());
        const int64_t tile = whole(a[1]);
        const bool transposed = truth(a[2]), both = truth(a[3]);
        const int32_t repeat = narrow(whole(a[5]));
        if (x.dim() != 2 || (tile != 1 && tile != MADDNESS_BLOCK) || repeat < 1) throw NotUsual();
        const Rows rx = rows_of(x);
        int64_t rows = rx.rows;
        const int32_t *source = nullptr;
        const float *factors = nullptr;
        if (a[4] != Py_None) {
            const at::Tensor &s = tensor(a[4]);
            if (s.dim() != 1 || s.scalar_type() != at::kInt || !s.is_contiguous() || s.device() != x.device()) throw NotUsual();
            rows = s.size(0);
            source = static_cast<const int32_t *>(s.data_ptr());
            if (a[6] != Py_None) {
                const at::Tensor &f = plain(a[6]);
                if (f.scalar_type() != at::kFloat || !f.is_contiguous() || f.numel() != rx.rows * repeat || f.device() != x.device()) throw NotUsual();
                factors = static_cast<const float *>(f.data_ptr());
            }
        } else if (a[6] != Py_None) {
            throw NotUsual();
        }
        void *stream = stream_of(Py_None);
        NewBlocks straight, turned;
        if (both || !transposed) straight = new_blocks(-1, rows, rx.cols, tile, x.device());
        if (both || transposed) turned = new_blocks(-1, rx.cols, rows, tile, x.device());
        auto bytes = [](const at::Tensor &t) { return t.defined() ? static_cast<uint8_t *>(t.data_ptr()) : nullptr; };
        const void *x_p = x.data_ptr();
        uint8_t *q = bytes(straight.q), *s = bytes(straight.scale), *qt = bytes(turned.q), *st = bytes(turned.scale);
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = maddness_quantise_blocks(x_p, code, 1, rows, rx.cols, rx.ld, 0, (int32_t)tile, source, rx.rows, repeat, factors, q,
                                      q ? straight.ld : 0, s, q ? straight.lds : 0, qt, qt ? turned.ld : 0, st, qt ? turned.lds : 0, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        PyObject *tuple = PyTuple_New(both ? 4 : 2);
        Py_ssize_t at = 0;
        for (const NewBlocks *b : {&straight, &turned}) {
            if (!b->q.defined()) continue;
            PyTuple_SET_ITEM(tuple, at++, THPVariable_Wrap(b->q));
            PyTuple_SET_ITEM(tuple, at++, THPVariable_Wrap(b->scale));
        }
        return tuple;
    });
}

// (a_is_blocks, A, B, offsets, by, source, repeat, out_dtype, out, workspace) -> out
PyObject *block_product(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 10) throw NotUsual();
        at::Device device(at::kCPU);
        maddness_block_matrix A{}, B{};
        int64_t experts = -1;
        if (truth(a[0])) {
            A = block_matrix(a[1], nullptr, &experts, &device);
            if (experts != -1) throw NotUsual();
        } else {
            const at::Tensor &x = plain(a[1]);
            const Rows r = rows_of(x);
            A.data = x.data_ptr();
            A.dtype = float_code(x.scalar_type());
            A.tile = 1;
            A.rows = r.rows;
            A.cols = r.cols;
            A.ld = r.ld;
            device = x.device();
        }
        B = block_matrix(a[2], &device, &experts);
        if (A.cols != B.cols) throw NotUsual();
        int32_t by = narrow(whole(a[4])), groups = 1;
        const int32_t *offsets = nullptr;
        if (by == MADDNESS_BY_CHOICE) {
            if (experts < 1) throw NotUsual();
            groups = narrow(experts);
        } else if (a[3] != Py_None) {
            const at::Tensor &o = tensor(a[3]);
            if (o.dim() != 1 || o.scalar_type() != at::kInt || !o.is_contiguous() || o.device() != device || o.size(0) < 2) throw NotUsual();
            groups = narrow(o.size(0) - 1);
            offsets = static_cast<const int32_t *>(o.data_ptr());
            if (by == MADDNESS_BY_ROWS ? experts != groups : experts != -1) throw NotUsual();
        } else {
            if (experts != -1 || by != MADDNESS_BY_ROWS) throw NotUsual();
            by = MADDNESS_DENSE;
        }
        int64_t rows = A.rows;
        const int32_t repeat = narrow(whole(a[6])), *source = nullptr;
        if (a[5] != Py_None) {
            const at::Tensor &s = tensor(a[5]);
            if ((by != MADDNESS_BY_ROWS && by != MADDNESS_BY_CHOICE) || s.dim() != 1 || s.scalar_type() != at::kInt || !s.is_contiguous() || s.device() != device || repeat < 1)
                throw NotUsual();
            rows = s.size(0);
            source = rows ? static_cast<const int32_t *>(s.data_ptr()) : offsets;      // (an empty one may have no address, and is not read)
        }
        void *stream = stream_of(Py_None);
        at::Tensor made, work;
        const at::ScalarType type = dtype_or(a[7], at::kBFloat16);
        void *out;
        int64_t ldo;
        int code;
        if (a[8] == Py_None) {
            code = float_code(type);
            const auto opt = at::TensorOptions().dtype(type).device(device);
            made = by == MADDNESS_BY_DEPTH ? at::empty({groups, A.rows, B.rows}, opt) : at::empty({rows, B.rows}, opt);
            out = made.data_ptr();
            ldo = std::max(B.rows, (int64_t)1);
        } else {
            const at::Tensor &o = plain(a[8]);
            if (by == MADDNESS_BY_DEPTH || o.device() != device || (a[7] != Py_None && o.scalar_type() != type)) throw NotUsual();
            const Rows r = rows_of(o);
            if (r.rows != rows || r.cols != B.rows) throw NotUsual();
            code = float_code(o.scalar_type());
            out = o.data_ptr();
            ldo = r.ld;
        }
        void *work_p = nullptr;
        size_t work_bytes = 0;
        if (a[9] != Py_None) {
            const at::Tensor &w = tensor(a[9]);
            if (w.scalar_type() != at::kByte || !w.is_contiguous() || w.device() != device) throw NotUsual();
            work_p = w.data_ptr();
            work_bytes = (size_t)w.numel();
        } else if ((work_bytes = maddness_block_product_workspace(A.rows, A.cols, by, A.dtype))) {
            work = at::empty({(int64_t)work_bytes}, at::TensorOptions().dtype(at::kByte).device(device));
            work_p = work.data_ptr();
        }
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = maddness_block_product(&A, &B, by, groups, offsets, source, rows, repeat, out, code, ldo, work_p, work_bytes, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        if (made.defined()) return THPVariable_Wrap(std::move(made));
        Py_INCREF(a[8]);
        return a[8];
    });
}

// (logits, k, sigmoid, bias, groups, kept, renormalise, factor) -> (ids, weights)
PyObject *route(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 8 || !PyFloat_CheckExact(a[7])) throw NotUsual();
        const at::Tensor &x = plain(a[0]);
        const int code = float_code(x.scalar_type());
        const Rows r = rows_of(x);
        const int32_t k = narrow(whole(a[1])), groups = narrow(whole(a[4])), kept = narrow(whole(a[5]));
        const bool sigmoid = truth(a[2]), renormalise = truth(a[6]);
        if (k < 1 || r.cols > MADDNESS_MAX_EXPERTS) throw NotUsual();
        const float *bias = flat_or_null<const float>(a[3], at::kFloat, {r.cols}, x.device());
        void *stream = stream_of(Py_None);
        const auto opt = at::TensorOptions().device(x.device());
        at::Tensor ids = at::empty({r.rows, k}, opt.dtype(at::kInt)), weights = at::empty({r.rows, k}, opt.dtype(at::kFloat));
        int32_t *ids_p = static_cast<int32_t *>(ids.data_ptr());
        float *weights_p = static_cast<float *>(weights.data_ptr());
        const void *x_p = x.data_ptr();
        const float factor = (float)PyFloat_AS_DOUBLE(a[7]);
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = maddness_route(x_p, code, r.rows, (int32_t)r.cols, r.ld, bias, sigmoid ? MADDNESS_SIGMOID : MADDNESS_SOFTMAX, groups, kept, k,
                            renormalise, factor, ids_p, weights_p, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        PyObject *tuple = PyTuple_New(2);
        PyTuple_SET_ITEM(tuple, 0, THPVariable_Wrap(std::move(ids)));
        PyTuple_SET_ITEM(tuple, 1, THPVariable_Wrap(std::move(weights)));
        return tuple;
    });
}

// (logits, ids, weights_gradient, sigmoid, renormalise, factor) -> gradient
PyObject *route_gradient(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 6 || !PyFloat_CheckExact(a[5])) throw NotUsual();
        const at::Tensor &x = plain(a[0]), &ids = tensor(a[1]);
        const int code = float_code(x.scalar_type());
        const Rows r = rows_of(x);
        if (ids.dim() != 2 || r.cols > MADDNESS_MAX_EXPERTS) throw NotUsual();
        const int32_t k = narrow(ids.size(1));
        const int32_t *ids_p = flat_or_null<const int32_t>(a[1], at::kInt, {r.rows, k}, x.device());
        const float *dw = flat_or_null<const float>(a[2], at::kFloat, {r.rows, k}, x.device());
        const bool sigmoid = truth(a[3]), renormalise = truth(a[4]);
        void *stream = stream_of(Py_None);
        at::Tensor out = at::empty({r.rows, r.cols}, x.options());
        const void *x_p = x.data_ptr();
        void *out_p = out.data_ptr();
        const float factor = (float)PyFloat_AS_DOUBLE(a[5]);
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = maddness_route_gradient(x_p, code, r.rows, (int32_t)r.cols, r.ld, sigmoid ? MADDNESS_SIGMOID : MADDNESS_SOFTMAX, k, renormalise, factor,
                                     ids_p, dw, out_p, r.cols, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        return THPVariable_Wrap(std::move(out));
    });
}

// (ids, experts, align) -> (offsets, counts, source, place)
PyObject *order(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 3) throw NotUsual();
        const at::Tensor &ids = tensor(a[0]);
        if (ids.scalar_type() != at::kInt || !ids.is_contiguous()) throw NotUsual();
        const int32_t E = narrow(whole(a[1])), align = narrow(whole(a[2]));
        if (E < 1 || E > MADDNESS_MAX_EXPERTS || align < 1) throw NotUsual();
        const int64_t slots = ids.numel(), capacity = maddness_order_capacity(slots, E, align);
        const int64_t work = ((int64_t)maddness_order_workspace(slots, E) + 3) / 4;
        void *stream = stream_of(Py_None);
        const auto opt = ids.options();
        // one piece of memory: source first, for its alignment
        at::Tensor all = at::empty({capacity + E + 1 + E + work}, opt), place = at::empty(ids.sizes(), opt);
        int32_t *base = static_cast<int32_t *>(all.data_ptr()), *place_p = static_cast<int32_t *>(place.data_ptr());
        const int32_t *ids_p = static_cast<const int32_t *>(ids.data_ptr());
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = maddness_order(ids_p, slots, E, align, base + capacity, base + capacity + E + 1, base, capacity, place_p, base + capacity + 2 * E + 1,
                            (size_t)work * 4, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        PyObject *tuple = PyTuple_New(4);
        PyTuple_SET_ITEM(tuple, 0, THPVariable_Wrap(all.narrow(0, capacity, E + 1)));
        PyTuple_SET_ITEM(tuple, 1, THPVariable_Wrap(all.narrow(0, capacity + E + 1, E)));
        PyTuple_SET_ITEM(tuple, 2, THPVariable_Wrap(all.narrow(0, 0, capacity)));
        PyTuple_SET_ITEM(tuple, 3, THPVariable_Wrap(std::move(place)));
        return tuple;
    });
}

// (y, place, weights, out_dtype, out) -> out
PyObject *combine(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 5) throw NotUsual();
        const at::Tensor &y = plain(a[0]), &slots = tensor(a[a[1] == Py_None ? 2 : 1]);
        const int code = float_code(y.scalar_type());
        const Rows r = rows_of(y);
        if (slots.dim() != 2 || a[4] != Py_None) throw NotUsual();
        const int64_t T = slots.size(0);
        const int32_t k = narrow(slots.size(1));
        const int32_t *place_p = flat_or_null<const int32_t>(a[1], at::kInt, {T, k}, y.device());
        const float *weights = flat_or_null<const float>(a[2], at::kFloat, {T, k}, y.device());
        const at::ScalarType type = dtype_or(a[3], y.scalar_type());
        const int out_code = float_code(type);
        void *stream = stream_of(Py_None);
        at::Tensor out = at::empty({T, r.cols}, y.options().dtype(type));
        const void *y_p = y.data_ptr();
        void *out_p = out.data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = maddness_combine(y_p, code, r.rows, r.cols, r.ld, place_p, weights, T, k, out_p, out_code, r.cols, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        return THPVariable_Wrap(std::move(out));
    });
}

// (gradient, y, place) -> weights_gradient
PyObject *combine_gradient(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 3) throw NotUsual();
        const at::Tensor &g = plain(a[0]), &y = plain(a[1]), &place = tensor(a[2]);
        const int code = float_code(g.scalar_type()), y_code = float_code(y.scalar_type());
        const Rows rg = rows_of(g), ry = rows_of(y);
        if (place.dim() != 2 || rg.cols != ry.cols || g.device() != y.device()) throw NotUsual();
        const int32_t k = narrow(place.size(1));
        const int32_t *place_p = flat_or_null<const int32_t>(a[2], at::kInt, {rg.rows, k}, y.device());
        void *stream = stream_of(Py_None);
        at::Tensor out = at::empty({rg.rows, k}, y.options().dtype(at::kFloat));
        const void *g_p = g.data_ptr(), *y_p = y.data_ptr();
        float *out_p = static_cast<float *>(out.data_ptr());
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = maddness_combine_gradient(g_p, code, rg.ld, y_p, y_code, ry.rows, ry.cols, ry.ld, place_p, rg.rows, k, out_p, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        return THPVariable_Wrap(std::move(out));
    });
}

// ---------------------------------------------------------------- 8-bit integers, layer norm, balance of experts, gradients' norm

// The current stream of the current device, which has to be the tensors' one.
void *stream_on(const at::Device &device)
{
    Ref current(PyObject_CallNoArgs(get_device));
    if (whole(current.p) != device.index()) throw NotUsual();
    Ref raw(PyObject_CallOneArg(get_stream, current.p));
    return reinterpret_cast<void *>(whole(raw.p));
}

at::Tensor fresh(at::IntArrayRef sizes, at::ScalarType type, const at::Device &device) { return at::empty(sizes, at::TensorOptions().dtype(type).device(device)); }

// n elements (n < 0: one, without dimensions) of a tensor's memory from the offset-th on, as a tensor of their own: results of one call that are small share an
// allocation (each would take 0.9 us).
at::Tensor part_of(const at::Tensor &all, int64_t offset, int64_t n)
{
    auto impl = c10::make_intrusive<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), all.dtype());
    impl->set_storage_offset(offset);
    if (n < 0) impl->set_sizes_contiguous(at::IntArrayRef());
    else impl->set_sizes_contiguous({n});
    return at::Tensor(std::move(impl));
}

// Memory for the time of a call, of the current device's current stream (a tensor of it takes 0.4 us more).
struct Scratch {
    c10::DataPtr memory;
    size_t bytes = 0;
    explicit Scratch(size_t n) : bytes(n)
    {
        if (n) memory = c10::GetAllocator(c10::DeviceType::CUDA)->allocate(n);
    }
    void *get() const { return memory.get(); }
};

float real(PyObject *o)
{
    if (!PyFloat_CheckExact(o)) throw NotUsual();
    return (float)PyFloat_AS_DOUBLE(o);
}

template <typename... T>
PyObject *tuple_of(const T &...t)
{
    PyObject *tuple = PyTuple_New(sizeof...(T));
    Py_ssize_t at = 0;
    (PyTuple_SET_ITEM(tuple, at++, THPVariable_Wrap(t)), ...);
    return tuple;
}

// An IntegerMatrix: what its constructor checks, as its tensors may have been replaced since.
maddness_integer_matrix integer_matrix(PyObject *o, const at::Device *device, at::Device *own)
{
    Ref q_ref(PyObject_GetAttr(o, s_q)), scale_ref(PyObject_GetAttr(o, s_scale));
    const at::Tensor &q = tensor(q_ref.p);
    if (q.dim() != 2 || q.scalar_type() != at::kChar || (device && q.device() != *device) || (q.size(1) > 1 && q.stride(1) != 1)) throw NotUsual();
    const at::Tensor &scale = flat(scale_ref.p, at::kFloat, {q.size(0)}, q.device());
    maddness_integer_matrix m{};
    m.data = q.data_ptr();
    m.dtype = MADDNESS_I8;
    m.rows = q.size(0);
    m.cols = q.size(1);
    m.ld = m.rows > 1 ? q.stride(0) : up(std::max(m.cols, q.stride(0)), 16);
    m.scale = static_cast<const float *>(scale.data_ptr());
    if (own) *own = q.device();
    return m;
}

struct NewIntegers {
    at::Tensor q, scale;
    int64_t ld;
};

NewIntegers new_integers(int64_t rows, int64_t cols, const at::Device &device)
{
    NewIntegers b;
    b.ld = up(cols, 16);
    b.q = fresh({rows, b.ld}, at::kChar, device);
    b.scale = fresh({rows}, at::kFloat, device);
    if (b.ld != cols) b.q = b.q.narrow(1, 0, cols);
    return b;
}

// (x) -> (q, scale)
PyObject *quantise_rows(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 1) throw NotUsual();
        const at::Tensor &x = plain(a[0]);
        const int code = float_code(x.scalar_type());
        const Rows r = rows_of(x);
        void *stream = stream_on(x.device());
        const NewIntegers out = new_integers(r.rows, r.cols, x.device());
        const void *x_p = x.data_ptr();
        int8_t *q = static_cast<int8_t *>(out.q.data_ptr());
        float *scale = static_cast<float *>(out.scale.data_ptr());
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = maddness_quantise_rows(x_p, code, r.rows, r.cols, r.ld, q, out.ld, scale, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        return tuple_of(out.q, out.scale);
    });
}

// (a_is_integers, A, B, bias, out_dtype, out, workspace) -> out
PyObject *integer_product(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 7) throw NotUsual();
        at::Device device(at::kCPU);
        maddness_integer_matrix A{};
        if (truth(a[0])) {
            A = integer_matrix(a[1], nullptr, &device);
        } else {
            const at::Tensor &x = plain(a[1]);
            const Rows r = rows_of(x);
            A.data = x.data_ptr();
            A.dtype = float_code(x.scalar_type());
            A.rows = r.rows;
            A.cols = r.cols;
            A.ld = r.ld;
            device = x.device();
        }
        const maddness_integer_matrix B = integer_matrix(a[2], &device, nullptr);
        if (A.cols != B.cols) throw NotUsual();
        const float *bias = flat_or_null<const float>(a[3], at::kFloat, {B.rows}, device);
        const at::ScalarType type = dtype_or(a[4], at::kBFloat16);
        void *stream = stream_on(device);
        at::Tensor made;
        void *out;
        int64_t ldo;
        int code;
        if (a[5] == Py_None) {
            code = float_code(type);
            made = fresh({A.rows, B.rows}, type, device);
            out = made.data_ptr();
            ldo = B.rows;
        } else {
            const at::Tensor &o = plain(a[5]);
            if (o.device() != device || (a[4] != Py_None && o.scalar_type() != type)) throw NotUsual();
            const Rows r = rows_of(o);
            if (r.rows != A.rows || r.cols != B.rows) throw NotUsual();
            code = float_code(o.scalar_type());
            out = o.data_ptr();
            ldo = r.ld;
        }
        const Scratch work(a[6] == Py_None ? maddness_integer_product_workspace(A.rows, A.cols, A.dtype) : 0);
        void *work_p = work.get();
        size_t work_bytes = work.bytes;
        if (a[6] != Py_None) {
            const at::Tensor &w = tensor(a[6]);
            if (w.scalar_type() != at::kByte || !w.is_contiguous() || w.device() != device) throw NotUsual();
            work_p = w.data_ptr();
            work_bytes = (size_t)w.numel();
        }
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = maddness_integer_product(&A, &B, bias, out, code, ldo, work_p, work_bytes, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        if (made.defined()) return THPVariable_Wrap(std::move(made));
        Py_INCREF(a[5]);
        return a[5];
    });
}

// A norm's weight or bias (or nullptr); its type has to be that of the other one.
const void *parameter(PyObject *o, int64_t cols, const at::Device &device, int *code)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = plain(o);
    const int c = float_code(t.scalar_type());
    if (t.dim() != 1 || t.size(0) != cols || !t.is_contiguous() || t.device() != device || (*code >= 0 && c != *code)) throw NotUsual();
    *code = c;
    return t.data_ptr();
}

// (x, weight, bias, eps, training, integer, out_dtype, out) -> out, or (out [or q, scale], mean, rstd), or (q, scale)
PyObject *layer_norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 8 || a[7] != Py_None) throw NotUsual();
        const at::Tensor &x = plain(a[0]);
        const int code = float_code(x.scalar_type());
        const Rows r = rows_of(x);
        int parameters = -1;
        const void *weight = parameter(a[1], r.cols, x.device(), &parameters), *bias = parameter(a[2], r.cols, x.device(), &parameters);
        const float eps = real(a[3]);
        const bool training = truth(a[4]), integer = truth(a[5]);
        const at::ScalarType type = dtype_or(a[6], x.scalar_type());
        const int out_code = integer ? (int)MADDNESS_I8 : float_code(type);
        void *stream = stream_on(x.device());
        at::Tensor y, mean, rstd;
        NewIntegers q;
        if (integer) q = new_integers(r.rows, r.cols, x.device());
        else y = fresh({r.rows, r.cols}, type, x.device());
        if (training) {
            const at::Tensor both = fresh({2, r.rows}, at::kFloat, x.device());
            mean = part_of(both, 0, r.rows);
            rstd = part_of(both, r.rows, r.rows);
        }
        const void *x_p = x.data_ptr();
        void *out = integer ? q.q.data_ptr() : y.data_ptr();
        const int64_t ldo = integer ? q.ld : r.cols;
        float *scale = integer ? static_cast<float *>(q.scale.data_ptr()) : nullptr;
        float *mean_p = training ? static_cast<float *>(mean.data_ptr()) : nullptr, *rstd_p = training ? static_cast<float *>(rstd.data_ptr()) : nullptr;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = maddness_layer_norm(x_p, code, r.rows, r.cols, r.ld, weight, bias, std::max(parameters, 0), eps, out, out_code, ldo, scale, mean_p, rstd_p, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        if (integer) return training ? tuple_of(q.q, q.scale, mean, rstd) : tuple_of(q.q, q.scale);
        return training ? tuple_of(y, mean, rstd) : THPVariable_Wrap(std::move(y));
    });
}

// (gradient, x, mean, rstd, weight, parameters) -> (dx, dweight, dbias)
PyObject *layer_norm_gradient(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 6) throw NotUsual();
        const at::Tensor &g = plain(a[0]), &x = plain(a[1]);
        const int g_code = float_code(g.scalar_type()), code = float_code(x.scalar_type());
        const Rows rg = rows_of(g), r = rows_of(x);
        if (rg.rows != r.rows || rg.cols != r.cols || g.device() != x.device()) throw NotUsual();
        const float *mean = static_cast<const float *>(flat(a[2], at::kFloat, {r.rows}, x.device()).data_ptr());
        const float *rstd = static_cast<const float *>(flat(a[3], at::kFloat, {r.rows}, x.device()).data_ptr());
        int parameter_code = -1;
        const void *weight = parameter(a[4], r.cols, x.device(), &parameter_code);
        const bool parameters = truth(a[5]);
        void *stream = stream_on(x.device());
        at::Tensor dx = fresh({r.rows, r.cols}, x.scalar_type(), x.device()), dweight, dbias;
        const Scratch work(parameters ? maddness_layer_norm_gradient_workspace(r.rows, r.cols) : 0);
        if (parameters) {
            const at::Tensor both = fresh({2, r.cols}, at::kFloat, x.device());
            dweight = part_of(both, 0, r.cols);
            dbias = part_of(both, r.cols, r.cols);
        }
        const void *g_p = g.data_ptr(), *x_p = x.data_ptr();
        void *dx_p = dx.data_ptr();
        float *dweight_p = parameters ? static_cast<float *>(dweight.data_ptr()) : nullptr, *dbias_p = parameters ? static_cast<float *>(dbias.data_ptr()) : nullptr;
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = maddness_layer_norm_gradient(g_p, g_code, rg.ld, x_p, code, r.rows, r.cols, r.ld, mean, rstd, weight, std::max(parameter_code, 0), dx_p, r.cols,
                                          dweight_p, dbias_p, work.get(), work.bytes, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        if (parameters) return tuple_of(dx, dweight, dbias);
        PyObject *tuple = PyTuple_New(3);
        PyTuple_SET_ITEM(tuple, 0, THPVariable_Wrap(std::move(dx)));
        for (int i = 1; i < 3; ++i) {
            Py_INCREF(Py_None);
            PyTuple_SET_ITEM(tuple, i, Py_None);
        }
        return tuple;
    });
}

// (logits, ids, sigmoid, factor) -> (loss, counts, push)
PyObject *balance(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 4) throw NotUsual();
        const at::Tensor &x = plain(a[0]), &ids = tensor(a[1]);
        const int code = float_code(x.scalar_type());
        const Rows r = rows_of(x);
        if (ids.dim() != 2 || r.cols < 1 || r.cols > MADDNESS_MAX_EXPERTS) throw NotUsual();
        const int32_t k = narrow(ids.size(1)), E = (int32_t)r.cols;
        if (k < 1) throw NotUsual();
        const int32_t *ids_p = flat_or_null<const int32_t>(a[1], at::kInt, {r.rows, k}, x.device());
        const bool sigmoid = truth(a[2]);
        const float factor = real(a[3]);
        void *stream = stream_on(x.device());
        const Scratch work(maddness_balance_workspace(r.rows, E));
        // (memory of one type: torch.save refuses tensors that share it with two)
        const at::Tensor all = fresh({E + 1}, at::kFloat, x.device()), counts = fresh({E}, at::kInt, x.device());
        const at::Tensor loss = part_of(all, 0, -1), push = part_of(all, 1, E);
        const void *x_p = x.data_ptr();
        float *loss_p = static_cast<float *>(loss.data_ptr()), *push_p = static_cast<float *>(push.data_ptr());
        int32_t *counts_p = static_cast<int32_t *>(counts.data_ptr());
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = maddness_balance(x_p, code, r.rows, E, r.ld, sigmoid ? MADDNESS_SIGMOID : MADDNESS_SOFTMAX, ids_p, k, factor, loss_p, counts_p, push_p,
                              work.get(), work.bytes, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        return tuple_of(loss, counts, push);
    });
}

// (logits, push, sigmoid, loss_gradient, add, out) -> gradient
PyObject *balance_gradient(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 6) throw NotUsual();
        const at::Tensor &x = plain(a[0]);
        const int code = float_code(x.scalar_type());
        const Rows r = rows_of(x);
        if (r.cols < 1 || r.cols > MADDNESS_MAX_EXPERTS) throw NotUsual();
        const float *push = static_cast<const float *>(flat(a[1], at::kFloat, {r.cols}, x.device()).data_ptr());
        const bool sigmoid = truth(a[2]);
        const float *times = nullptr;
        if (a[3] != Py_None) {
            const at::Tensor &t = plain(a[3]);
            if (t.scalar_type() != at::kFloat || t.numel() != 1 || t.device() != x.device()) throw NotUsual();
            times = static_cast<const float *>(t.data_ptr());
        }
        auto like = [&](PyObject *o, int64_t *ld) -> void * {
            const at::Tensor &t = plain(o);
            const Rows rt = rows_of(t);
            if (t.scalar_type() != x.scalar_type() || rt.rows != r.rows || rt.cols != r.cols || t.device() != x.device()) throw NotUsual();
            *ld = rt.ld;
            return t.data_ptr();
        };
        int64_t lda = 0, ldd = r.cols;
        const void *add = a[4] == Py_None ? nullptr : like(a[4], &lda);
        at::Tensor made;
        void *out, *stream = stream_on(x.device());
        if (a[5] == Py_None) {
            made = fresh({r.rows, r.cols}, x.scalar_type(), x.device());
            out = made.data_ptr();
        } else {
            out = like(a[5], &ldd);
        }
        const void *x_p = x.data_ptr();
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = maddness_balance_gradient(x_p, code, r.rows, (int32_t)r.cols, r.ld, sigmoid ? MADDNESS_SIGMOID : MADDNESS_SOFTMAX, push, times, add, lda, out, ldd, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        if (made.defined()) return THPVariable_Wrap(std::move(made));
        Py_INCREF(a[5]);
        return a[5];
    });
}

// (tensors, max_norm or None, norm, out) -> norm: scales the tensors where there is a max_norm
PyObject *clip_gradients(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return usual([&]() -> PyObject * {
        if (n != 4 || !PyList_CheckExact(a[0]) || (a[3] != Py_None && !PyList_CheckExact(a[3]))) throw NotUsual();
        const Py_ssize_t count = PyList_GET_SIZE(a[0]);
        if (count == 0 || (a[3] != Py_None && PyList_GET_SIZE(a[3]) != count)) throw NotUsual();
        const bool scales = a[1] != Py_None;
        const float max_norm = scales ? real(a[1]) : 0.0f;
        std::vector<maddness_tensor> table((size_t)count);
        const at::Device device = tensor(PyList_GET_ITEM(a[0], 0)).device();
        for (Py_ssize_t i = 0; i < count; ++i) {
            const at::Tensor &t = plain(PyList_GET_ITEM(a[0], i));
            if (t.device() != device || !t.is_non_overlapping_and_dense()) throw NotUsual();
            maddness_tensor &to = table[(size_t)i];
            to.data = to.out = t.data_ptr();
            to.count = t.numel();
            to.dtype = to.out_dtype = float_code(t.scalar_type());
            if (!scales || a[3] == Py_None) continue;
            const at::Tensor &o = plain(PyList_GET_ITEM(a[3], i));
            if (o.device() != device || o.sizes() != t.sizes() || o.strides() != t.strides()) throw NotUsual();
            to.out = o.data_ptr();
            to.out_dtype = float_code(o.scalar_type());
        }
        void *stream = stream_on(device);
        at::Tensor norm;
        const bool given = a[2] != Py_None;
        const Scratch work(given ? 0 : maddness_gradient_norm_workspace());
        if (given) {
            norm = plain(a[2]);
            if (norm.scalar_type() != at::kFloat || norm.numel() != 1 || norm.device() != device) throw NotUsual();
        } else {
            norm = fresh({}, at::kFloat, device);
        }
        float *norm_p = static_cast<float *>(norm.data_ptr());
        int rc;
        Py_BEGIN_ALLOW_THREADS
        rc = scales ? maddness_clip_gradients(table.data(), count, max_norm, norm_p, given, work.get(), work.bytes, stream)
                    : maddness_gradient_norm(table.data(), count, norm_p, work.get(), work.bytes, stream);
        Py_END_ALLOW_THREADS
        if (rc != MADDNESS_OK) return int_status(rc);
        if (!given) return THPVariable_Wrap(std::move(norm));
        Py_INCREF(a[2]);
        return a[2];
    });
}

// Tensors are read by the layout of the torch, and objects by that of the Python, that this was built with: with others it is an
// ImportError, also where every symbol is found.
bool built_for_these()
{
    PyObject *torch = PyImport_ImportModule("torch");
    PyObject *version = torch ? PyObject_GetAttrString(torch, "__version__") : nullptr;
    const char *have = version ? PyUnicode_AsUTF8(version) : nullptr;
    char python[32];
    std::snprintf(python, sizeof python, "%d.%d.", PY_MAJOR_VERSION, PY_MINOR_VERSION);
    const bool same = have && std::strcmp(have, MADDNESS_TORCH_VERSION) == 0 && std::strncmp(Py_GetVersion(), python, std::strlen(python)) == 0;
    if (!same && !PyErr_Occurred())
        PyErr_Format(PyExc_ImportError, "built for torch %s and Python %s, this is torch %s and Python %s", MADDNESS_TORCH_VERSION, PY_VERSION,
                     have, Py_GetVersion());
    Py_XDECREF(version);
    Py_XDECREF(torch);
    return same;
}

PyMethodDef methods[] = {
    {"encode_scan", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(encode_scan)), METH_FASTCALL, nullptr},
    {"encode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(encode)), METH_FASTCALL, nullptr},
    {"scan", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(scan)), METH_FASTCALL, nullptr},
    {"build_luts", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(build_luts)), METH_FASTCALL, nullptr},
    {"quantise_blocks", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(quantise_blocks)), METH_FASTCALL, nullptr},
    {"block_product", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(block_product)), METH_FASTCALL, nullptr},
    {"route", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(route)), METH_FASTCALL, nullptr},
    {"route_gradient", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(route_gradient)), METH_FASTCALL, nullptr},
    {"order", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(order)), METH_FASTCALL, nullptr},
    {"combine", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(combine)), METH_FASTCALL, nullptr},
    {"combine_gradient", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(combine_gradient)), METH_FASTCALL, nullptr},
    {"quantise_rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(quantise_rows)), METH_FASTCALL, nullptr},
    {"integer_product", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(integer_product)), METH_FASTCALL, nullptr},
    {"layer_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(layer_norm)), METH_FASTCALL, nullptr},
    {"layer_norm_gradient", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(layer_norm_gradient)), METH_FASTCALL, nullptr},
    {"balance", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(balance)), METH_FASTCALL, nullptr},
    {"balance_gradient", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(balance_gradient)), METH_FASTCALL, nullptr},
    {"clip_gradients", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(clip_gradients)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "maddness_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_maddness_binding()
{
    s_split_dims = PyUnicode_InternFromString("split_dims");
    s_thresholds = PyUnicode_InternFromString("thresholds");
    s_prototypes = PyUnicode_InternFromString("prototypes");
    s_C = PyUnicode_InternFromString("C");
    s_D = PyUnicode_InternFromString("D");
    s_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    s_q = PyUnicode_InternFromString("q");
    s_scale = PyUnicode_InternFromString("scale");
    s_tile = PyUnicode_InternFromString("tile");
    if (!built_for_these()) return nullptr;
    PyObject *torch_c = PyImport_ImportModule("torch._C");
    if (!torch_c) return nullptr;
    get_stream = PyObject_GetAttrString(torch_c, "_cuda_getCurrentRawStream");
    get_device = PyObject_GetAttrString(torch_c, "_cuda_getDevice");
    Py_DECREF(torch_c);
    if (!get_stream || !get_device) return nullptr;
    return PyModule_Create(&module);
}
