// Arguments of the library's calls from Python: device addresses of checked tensors, whole job arrays, and the calls of cnr_lm.h.
//
// A call of the library is one or two launches of a few microseconds, and what its caller in Python does beforehand
// is checks of up to twelve tensors (of dozens for a batch): four attributes of each and an object for its
// address, 0.26 to 0.34 us apiece in Python, 0.06 here.  An iteration's mark of eight tables 19 us a call with the checks in
// Python, small checkpoints 50 us.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <initializer_list>

namespace {

constexpr Py_ssize_t kJobFields = 16;  // of cnr_table_job, each 64 bits

PyObject *general = nullptr;  // address() of anything but plain tensors and parameters

// Device address of a contiguous GPU tensor of the given dtype (None: any); 0 for None.  False: a Python error is set.
bool address_of(PyObject *t, PyObject *dtype, PyObject *name, unsigned long long &out) {
    out = 0;
    if (t == Py_None) return true;
    if (!THPVariable_CheckExact(t)) {  // subclasses answer for themselves; the rest is refused there
        THPObjectPtr r(PyObject_CallFunctionObjArgs(general, t, dtype, name, nullptr));
        if (!r) return false;
        out = PyLong_AsUnsignedLongLong(r.get());
        return !PyErr_Occurred();
    }
    const at::Tensor &v = THPVariable_Unpack(t);
    if (!v.is_cuda()) {
        PyErr_Format(PyExc_TypeError, "%S must be a tensor on the GPU", name);
        return false;
    }
    if (dtype != Py_None) {
        if (!THPDtype_Check(dtype)) {
            PyErr_SetString(PyExc_TypeError, "dtype must be a torch.dtype or None");
            return false;
        }
        if (v.scalar_type() != reinterpret_cast<THPDtype *>(dtype)->scalar_type) {
            PyObject *got = PyObject_GetAttrString(t, "dtype");
            if (got) PyErr_Format(PyExc_TypeError, "%S must be %S, got %S", name, dtype, got);
            Py_XDECREF(got);
            return false;
        }
    }
    if (!v.is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%S must be contiguous", name);
        return false;
    }
    out = (unsigned long long)(uintptr_t)v.data_ptr();
    return true;
}

PyObject *address(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 3) {
        PyErr_SetString(PyExc_TypeError, "address(tensor, dtype, name)");
        return nullptr;
    }
    unsigned long long p;
    return address_of(args[0], args[1], args[2], p) ? PyLong_FromUnsignedLongLong(p) : nullptr;
    END_HANDLE_TH_ERRORS
}

// A field of a job: a number where `kind` is the type int (anything with __index__), else an address, of a tensor of dtype `kind` or for
// None or the number 0, a field that the call does not read.
bool field(PyObject *v, PyObject *kind, PyObject *name, unsigned long long &out) {
    if (kind == reinterpret_cast<PyObject *>(&PyLong_Type)) {
        if (PyLong_CheckExact(v)) {
            out = PyLong_AsUnsignedLongLong(v);
        } else {
            THPObjectPtr index(PyNumber_Index(v));
            if (!index) return false;
            out = PyLong_AsUnsignedLongLong(index.get());
        }
        return out != ~0ull || !PyErr_Occurred();
    }
    out = 0;
    if (v == Py_None) return true;
    if (PyLong_CheckExact(v)) {
        int overflow;
        if (PyLong_AsLongLongAndOverflow(v, &overflow) == 0 && !overflow) return true;
    }
    return address_of(v, kind, name, out);
}

// pack_jobs(rows, kinds, names): rows of sixteen fields, the struct's in order; the bytes of the array.
PyObject *pack_jobs(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != 3 || !PyList_Check(args[0]) || !PyTuple_Check(args[1]) || !PyTuple_Check(args[2]) ||
        PyTuple_GET_SIZE(args[1]) != kJobFields || PyTuple_GET_SIZE(args[2]) != kJobFields) {
        PyErr_SetString(PyExc_TypeError, "pack_jobs(list of rows, kinds, names)");
        return nullptr;
    }
    const Py_ssize_t rows = PyList_GET_SIZE(args[0]);
    THPObjectPtr bytes(PyBytes_FromStringAndSize(nullptr, rows * kJobFields * 8));  // given back if a tensor throws, too
    if (!bytes) return nullptr;
    for (Py_ssize_t i = 0; i < rows; ++i) {
        // the list can change hands while a subclass answers: its length is looked at again, the row is held
        PyObject *at = i < PyList_GET_SIZE(args[0]) ? PyList_GET_ITEM(args[0], i) : nullptr;
        if (!at || !PyTuple_Check(at) || PyTuple_GET_SIZE(at) != kJobFields) {
            PyErr_SetString(PyExc_TypeError, "a job has sixteen fields");
            return nullptr;
        }
        Py_INCREF(at);
        THPObjectPtr row(at);
        for (Py_ssize_t f = 0; f < kJobFields; ++f) {
            unsigned long long x;
            if (!field(PyTuple_GET_ITEM(at, f), PyTuple_GET_ITEM(args[1], f), PyTuple_GET_ITEM(args[2], f), x)) return nullptr;
            memcpy(PyBytes_AS_STRING(bytes.get()) + (i * kJobFields + f) * 8, &x, 8);
        }
    }
    return bytes.release();
    END_HANDLE_TH_ERRORS
}

// ---- the calls of a BatchCheckpointer ------------------------------------------------------------------
// batch_jobs(checkpointers, stage, tensors, outputs): the bytes of the job array of one stage of a batch, in one step from the objects that own
// the buffers; for the mark (bytes, index type).  Only what is in order in every respect is taken here: None is returned for anything else,
// and the caller's general way answers or refuses it.  Nothing is kept from one call to the next.  (An iteration's mark of eight tables as
// called 8.7 -> 6.9 us, of which the GPU is busy for 6.5; the five calls of a small checkpoint 26 -> 23 us on the host, fifteen of them the launches.)
enum Stage { kClear, kMark, kCompact, kRows };
const char *const kNames[] = {"n_rows", "dim", "capacity", "bitmap", "mark_scratch", "row_ids", "n_dirty", "scratch", "scale", "bias", "packed", "bits", "row_min", "row_max"};
enum Name { kNRows, kDim, kCapacity, kBitmap, kMarkScratch, kRowIds, kNDirty, kScratch, kScale, kBias, kPacked, kBits, kRowMin, kRowMax, kNameCount };
PyObject *names[kNameCount];

// The fields of cnr_table_job, in order.
enum Field { fTable, fNRows, fBitmap, fIndices, fNIndices, fMarkScratch, fRowIds, fCapacity, fNDirty, fScratch, fScale, fBias, fRowMin, fRowMax, fCodes, fPacked };

bool number(PyObject *owner, Name name, unsigned long long &out) {
    THPObjectPtr v(PyObject_GetAttr(owner, names[name]));
    if (!v || !PyLong_CheckExact(v.get())) return false;
    int overflow;
    const long long x = PyLong_AsLongLongAndOverflow(v.get(), &overflow);
    out = (unsigned long long)x;
    return !overflow && x >= 0;
}
// Address of a plain contiguous GPU tensor of this type (Undefined: any) with at least `least` elements.
bool plain(PyObject *v, at::ScalarType type, unsigned long long least, unsigned long long &out, unsigned long long *count = nullptr) {
    if (!THPVariable_CheckExact(v)) return false;
    const at::Tensor &t = THPVariable_Unpack(v);
    if (!t.is_cuda() || (type != at::ScalarType::Undefined && t.scalar_type() != type) || !t.is_contiguous()) return false;
    const unsigned long long n = (unsigned long long)t.numel();
    if (n < least) return false;
    if (count) *count = n;
    out = (unsigned long long)(uintptr_t)t.data_ptr();
    return true;
}
bool tensor(PyObject *owner, Name name, at::ScalarType type, bool may_be_none, unsigned long long least, unsigned long long &out) {
    THPObjectPtr v(PyObject_GetAttr(owner, names[name]));
    if (!v) return false;
    if (v.get() == Py_None) return may_be_none;  // out stays 0
    return plain(v.get(), type, least, out);
}
PyObject *item(PyObject *seq, Py_ssize_t i) {  // borrowed, of a list or a tuple
    if (PyList_CheckExact(seq)) return i < PyList_GET_SIZE(seq) ? PyList_GET_ITEM(seq, i) : nullptr;
    if (PyTuple_CheckExact(seq)) return i < PyTuple_GET_SIZE(seq) ? PyTuple_GET_ITEM(seq, i) : nullptr;
    return nullptr;
}
bool job(PyObject *owner, long stage, PyObject *t, PyObject *o, unsigned long long (&f)[kJobFields], at::ScalarType &index_type) {
    constexpr at::ScalarType i32 = at::kInt, i64 = at::kLong, f32 = at::kFloat, u8 = at::kByte, any = at::ScalarType::Undefined;
    if (!number(owner, kNRows, f[fNRows])) return false;
    if (stage != kRows && !tensor(owner, kBitmap, i32, false, 0, f[fBitmap])) return false;
    if (stage == kMark) {
        if (!tensor(owner, kMarkScratch, any, true, 0, f[fMarkScratch])) return false;
        if (t == Py_None) return true;
        if (!plain(t, any, 0, f[fIndices], &f[fNIndices])) return false;
        const at::ScalarType type = THPVariable_Unpack(t).scalar_type();
        if ((type != i32 && type != i64) || (index_type != any && index_type != type)) return false;
        index_type = type;
        return true;
    }
    if (stage == kClear) return true;
    if (!tensor(owner, kRowIds, i32, false, 0, f[fRowIds]) || !number(owner, kCapacity, f[fCapacity]) || !tensor(owner, kNDirty, i64, false, 0, f[fNDirty])) return false;
    if (stage == kCompact) return tensor(owner, kScratch, any, false, 0, f[fScratch]);
    unsigned long long dim, bits;
    if (!number(owner, kDim, dim) || !number(o, kBits, bits)) return false;
    if ((bits != 2 && bits != 3 && bits != 4 && bits != 8) || dim == 0 || dim > 1u << 20 || dim * bits % 8 || f[fNRows] >> 32 || f[fCapacity] >> 32) return false;
    const unsigned long long cap = f[fCapacity] ? f[fCapacity] : 1;
    return plain(t, f32, f[fNRows] * dim, f[fTable]) && tensor(o, kScale, f32, false, cap, f[fScale]) && tensor(o, kBias, f32, false, cap, f[fBias]) &&
           tensor(o, kRowMin, f32, true, 0, f[fRowMin]) && tensor(o, kRowMax, f32, true, 0, f[fRowMax]) &&
           tensor(o, kPacked, u8, false, cap * (dim * bits / 8), f[fPacked]);
}
PyObject *batch_jobs(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 4 || !PyList_CheckExact(args[0]) || !PyLong_CheckExact(args[1])) Py_RETURN_NONE;
    const long stage = PyLong_AsLong(args[1]);
    const Py_ssize_t rows = PyList_GET_SIZE(args[0]);
    THPObjectPtr bytes(PyBytes_FromStringAndSize(nullptr, rows * kJobFields * 8));
    if (!bytes) return nullptr;
    at::ScalarType index_type = at::ScalarType::Undefined;
    bool good = stage >= kClear && stage <= kRows;
    try {
        for (Py_ssize_t i = 0; i < rows && good; ++i) {
            // held: an attribute of an unusual object can run code that takes them out of their lists
            PyObject *owner = item(args[0], i), *t = stage == kMark || stage == kRows ? item(args[2], i) : Py_None, *o = stage == kRows ? item(args[3], i) : Py_None;
            if (!owner || !t || !o) {
                good = false;
                break;
            }
            Py_INCREF(owner);
            Py_INCREF(t);
            Py_INCREF(o);
            THPObjectPtr hold_owner(owner), hold_t(t), hold_o(o);
            unsigned long long f[kJobFields] = {};
            good = job(owner, stage, t, o, f, index_type);
            memcpy(PyBytes_AS_STRING(bytes.get()) + i * kJobFields * 8, f, sizeof(f));
        }
        // look-ups beyond the last table are not marked, but none may be of another type
        if (stage == kMark)
            for (Py_ssize_t i = rows; good; ++i) {
                PyObject *t = item(args[2], i);
                if (!t) break;
                good = t == Py_None || (THPVariable_CheckExact(t) && THPVariable_Unpack(t).scalar_type() == index_type);
            }
    } catch (...) {  // a tensor that has no address; the general way meets and reports it
        good = false;
    }
    if (!good || (stage == kMark && index_type == at::ScalarType::Undefined)) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    if (stage != kMark) return bytes.release();
    return Py_BuildValue("(NO)", bytes.release(), index_type == at::kInt ? Py_False : Py_True);
}

// ---- the calls of the operators for language models ------------------------------------------------------
// quantize_blocks, block_product, count_tokens and adjust_logits take what lm_binding's functions of these names take, in order, and make the library's call: its status is returned.  As above only what is in order is taken and None says that the general way
// has to look.  (32 x 2048 quantized as called 8.4 -> 6.4 us, 8 x 50257 logits adjusted 8.9 -> 5.2, one token of 256 sequences counted 6.2 -> 4.6.)

constexpr unsigned long long kBlock = 128, kMaxSize = 2147483647;
struct LmCalls {
    int (*quantize)(void *, const void *, int, uint64_t, uint64_t, uint64_t, int, int, void *, void *, void *, void *, void *);
    size_t (*workspace)(const void *, uint64_t, uint64_t, uint64_t);
    int (*product)(void *, const void *, const void *, int, uint64_t, const void *, const void *, int, uint64_t, uint64_t, int, void *, int, uint64_t, int, void *, void *);
    int (*count)(void *, void *, void *, uint64_t, uint64_t, const void *, uint64_t, int, const void *, const void *, uint64_t, int, int, void *);
    int (*adjust)(void *, const void *, uint64_t, void *, uint64_t, int, uint64_t, uint64_t, const void *, void *);
} lm;
PyObject *value_name = nullptr;  // "value"
PyObject *stream_of = nullptr;   // the handle of a stream, or of the current one for None

void *pointer(unsigned long long p) { return reinterpret_cast<void *>((uintptr_t)p); }

// Arguments one after the other, until one of them is not in order.
struct Arguments {
    PyObject *const *args;
    bool good;
    Arguments(PyObject *const *a, Py_ssize_t n, Py_ssize_t expected) : args(a), good(n == expected) {}
    PyObject *next() { return *args++; }
    void require(bool b) { good = good && b; }
    unsigned long long natural(unsigned long long limit = kMaxSize) {  // a number from 0 to `limit`, or a truth value
        PyObject *v = next();
        if (!good || !PyLong_Check(v)) return good = false, 0;
        int overflow;
        const long long x = PyLong_AsLongLongAndOverflow(v, &overflow);
        require(!overflow && x >= 0 && (unsigned long long)x <= limit);
        return (unsigned long long)x;
    }
    void *stream() {  // of a stream or None: its handle, asked for when all else is in order
        PyObject *v = next();
        if (!good) return nullptr;
        THPObjectPtr handle(PyObject_CallFunctionObjArgs(stream_of, v, nullptr));
        if (!handle || !PyLong_CheckExact(handle.get())) return good = false, nullptr;
        return PyLong_AsVoidPtr(handle.get());
    }
    void *context() {  // a ctypes.c_void_p that is not NULL
        PyObject *v = next();
        if (!good) return nullptr;
        THPObjectPtr number(PyObject_GetAttr(v, value_name));
        if (!number || !PyLong_CheckExact(number.get())) return good = false, nullptr;
        return PyLong_AsVoidPtr(number.get());
    }
    // Address of a list of at least `least` elements, 0 for None where that may be.
    unsigned long long list(at::ScalarType type, unsigned long long least, bool may_be_none = true, unsigned long long *count = nullptr) {
        PyObject *v = next();
        unsigned long long at = 0;
        if (good && (v != Py_None || !may_be_none)) good = plain(v, type, least, at, count);
        return at;
    }
    bool none() const { return *args == Py_None; }
    // A matrix of one of the three types with contiguous rows.
    struct Matrix {
        unsigned long long at, rows, columns, stride, element;
        int type;
    };
    Matrix matrix() {
        PyObject *v = next();
        Matrix m = {};
        if (!good || !THPVariable_CheckExact(v)) return good = false, m;
        const at::Tensor &t = THPVariable_Unpack(v);
        if (!t.is_cuda() || t.dim() != 2) return good = false, m;
        switch (t.scalar_type()) {
            case at::kFloat: m.type = 0, m.element = 4; break;
            case at::kBFloat16: m.type = 1, m.element = 2; break;
            case at::kHalf: m.type = 2, m.element = 2; break;
            default: return good = false, m;
        }
        m.rows = (unsigned long long)t.size(0), m.columns = (unsigned long long)t.size(1);
        require(t.stride(1) == 1 || m.columns <= 1);
        require(m.rows <= 1 || (t.stride(0) >= 0 && (unsigned long long)t.stride(0) >= m.columns));
        m.stride = m.rows <= 1 ? m.columns : (unsigned long long)t.stride(0);
        m.at = (unsigned long long)(uintptr_t)t.data_ptr();
        return m;
    }
    // Codes and scales of a blocked matrix.
    struct Blocked {
        void *codes, *scale;
    };
    Blocked blocked(unsigned long long n_rows, unsigned long long dim, unsigned long long kind, unsigned long long scale_type) {
        require(n_rows <= kMaxSize && dim <= kMaxSize);
        const unsigned long long across = (dim + kBlock - 1) / kBlock, down = (n_rows + kBlock - 1) / kBlock;
        Blocked b;
        b.codes = pointer(list(at::kByte, n_rows * across * kBlock, false));
        b.scale = pointer(list(scale_type ? at::kFloat : at::kByte, across * (kind ? down : down * kBlock), false));
        return b;
    }
};

// `written`: the call's results.  Autograd is told, as of torch's operations in place: what a graph has saved of them is not taken for
// unchanged.
template <typename Call>
PyObject *called(const Call &call, std::initializer_list<PyObject *> written) {
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = call();
    Py_END_ALLOW_THREADS
    for (PyObject *v : written) {
        if (status != 0 || !THPVariable_CheckExact(v)) continue;
        const at::Tensor &t = THPVariable_Unpack(v);
        if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    }
    return PyLong_FromLong(status);
}
PyObject *not_taken() {
    PyErr_Clear();
    Py_RETURN_NONE;
}

// (ctx, x, kind, scale_type, codes, scale, codes_t, scale_t, stream)
PyObject *quantize_blocks(PyObject *, PyObject *const *args, Py_ssize_t n) {
    try {
        Arguments a(args, n, 9);
        if (!a.good || !lm.quantize) return not_taken();
        void *ctx = a.context();
        const Arguments::Matrix x = a.matrix();
        const int kind = (int)a.natural(1), scale_type = (int)a.natural(1);
        Arguments::Blocked out = {}, out_t = {};
        if (a.none() && a.args[1] == Py_None)
            a.args += 2;
        else
            out = a.blocked(x.rows, x.columns, kind, scale_type);
        if (a.good && a.none() && a.args[1] == Py_None)
            a.args += 2;
        else if (a.good)
            out_t = a.blocked(x.columns, x.rows, kind, scale_type);
        if (!a.good) return not_taken();
        void *stream = a.stream();
        if (!a.good) return not_taken();
        return called([&] { return lm.quantize(ctx, pointer(x.at), x.type, x.rows, x.columns, x.stride, kind, scale_type, out.codes, out.scale, out_t.codes, out_t.scale, stream); },
                      {args[4], args[5], args[6], args[7]});
    } catch (...) {
        return not_taken();
    }
}

// (ctx, a_codes, a_scale, a_kind, m, b_codes, b_scale, b_kind, n, k, out, accumulate, workspace, stream)
PyObject *block_product(PyObject *, PyObject *const *args, Py_ssize_t count) {
    try {
        Arguments a(args, count, 14);
        if (!a.good || !lm.product) return not_taken();
        void *ctx = a.context();
        // sizes come after what they are the sizes of
        Arguments sizes(args + 3, 2, 2);
        const int a_kind = (int)sizes.natural(1);
        const unsigned long long m = sizes.natural();
        sizes.args = args + 7;
        const int b_kind = (int)sizes.natural(1);
        const unsigned long long n = sizes.natural(), k = sizes.natural();
        if (!a.good || !sizes.good || !THPVariable_CheckExact(args[2])) return not_taken();
        const int scale_type = THPVariable_Unpack(args[2]).scalar_type() == at::kFloat;
        const Arguments::Blocked x = a.blocked(m, k, a_kind, scale_type);
        a.args = args + 5;
        const Arguments::Blocked y = a.blocked(n, k, b_kind, scale_type);
        a.args = args + 10;
        const Arguments::Matrix out = a.matrix();
        a.require(out.rows >= m && out.columns >= n);
        const int accumulate = (int)a.natural(1);
        if (!a.good) return not_taken();
        void *workspace = nullptr;
        if (!a.none()) {
            if (!THPVariable_CheckExact(*a.args)) return not_taken();
            const at::Tensor &w = THPVariable_Unpack(*a.args);
            a.require((unsigned long long)w.numel() * w.element_size() >= lm.workspace(ctx, m, n, k));
        }
        workspace = pointer(a.list(at::ScalarType::Undefined, 0));
        void *stream = a.stream();
        if (!a.good) return not_taken();
        return called([&] {
            return lm.product(ctx, x.codes, x.scale, a_kind, m, y.codes, y.scale, b_kind, n, k, scale_type, pointer(out.at), out.type, out.stride, accumulate, workspace, stream);
        }, {args[10]});
    } catch (...) {
        return not_taken();
    }
}

// (ctx, seen, counts, n_slots, vocab, tokens, offsets, slots, prompt, restart, stream)
PyObject *count_tokens(PyObject *, PyObject *const *args, Py_ssize_t count) {
    try {
        Arguments a(args, count, 11);
        if (!a.good || !lm.count) return not_taken();
        Arguments sizes(args + 3, 2, 2);
        const unsigned long long n_slots = sizes.natural(), vocab = sizes.natural();
        void *ctx = a.context();
        if (!a.good || !sizes.good) return not_taken();
        void *seen = pointer(a.list(at::kInt, n_slots * ((vocab + 31) / 32))), *counts = pointer(a.list(at::kInt, n_slots * vocab));
        a.args = args + 5;
        if (!THPVariable_CheckExact(*a.args)) return not_taken();
        const at::ScalarType type = THPVariable_Unpack(*a.args).scalar_type();
        a.require(type == at::kInt || type == at::kLong);
        unsigned long long n_tokens = 0, n = 0;
        void *tokens = pointer(a.list(type, 0, false, &n_tokens));
        const bool listed = !a.none();
        void *offsets = pointer(a.list(at::kLong, 1, true, &n));
        n = listed ? n - 1 : n_tokens;
        void *slots = pointer(a.list(at::kInt, n));
        const int prompt = (int)a.natural(1), restart = (int)a.natural(1);
        void *stream = a.stream();
        if (!a.good) return not_taken();
        return called([&] { return lm.count(ctx, seen, counts, n_slots, vocab, tokens, n_tokens, type == at::kLong, offsets, slots, n, prompt, restart, stream); }, {args[1], args[2]});
    } catch (...) {
        return not_taken();
    }
}

// (ctx, logits, out, seen, counts, n_slots, slots, repetition, frequency, presence, bias_offsets, bias_tokens, bias_values, masks, n_masks, mask_of, stream)
PyObject *adjust_logits(PyObject *, PyObject *const *args, Py_ssize_t count) {
    try {
        Arguments a(args, count, 17);
        if (!a.good || !lm.adjust) return not_taken();
        void *ctx = a.context();
        const Arguments::Matrix from = a.matrix(), to = a.matrix();
        a.require(from.rows == to.rows && from.columns == to.columns && from.type == to.type);
        if (!a.good) return not_taken();
        const unsigned long long n = from.rows, vocab = from.columns, words = (vocab + 31) / 32;
        a.require(n <= kMaxSize && vocab <= kMaxSize && n > 0);
        a.require(to.at == from.at || to.at >= from.at + ((n - 1) * from.stride + vocab) * from.element ||
                  from.at >= to.at + ((n - 1) * to.stride + vocab) * to.element);
        Arguments sizes(args + 5, 1, 1);
        const unsigned long long n_slots = sizes.natural();
        sizes.args = args + 14;
        const unsigned long long n_masks = sizes.natural();
        if (!a.good || !sizes.good) return not_taken();
        unsigned long long w[14], values = 0, biases = 0;  // cnr_adjustments, field by field
        w[0] = a.list(at::kInt, n_slots * words), w[1] = a.list(at::kInt, n_slots * vocab);
        w[2] = n_slots;
        a.next();
        w[3] = a.list(at::kInt, n);
        for (int i = 4; i < 7; ++i) w[i] = a.list(at::kFloat, n);
        const bool biased = !a.none();
        w[7] = a.list(at::kLong, n + 1);
        w[8] = a.list(at::kInt, 0, true, &biases), w[9] = a.list(at::kFloat, 0, true, &values);
        a.require(!biased || (args[11] != Py_None && args[12] != Py_None && biases == values));
        w[10] = biased ? biases : 0;
        w[11] = a.list(at::kInt, n_masks * words);
        w[12] = n_masks;
        a.next();
        w[13] = a.list(at::kInt, n);
        void *stream = a.stream();
        if (!a.good) return not_taken();
        return called([&] { return lm.adjust(ctx, pointer(from.at), from.stride, pointer(to.at), to.stride, from.type, n, vocab, w, stream); }, {args[2]});
    } catch (...) {
        return not_taken();
    }
}

// set_lm(quantize, workspace, product, count, adjust, stream_of): addresses of the library's functions, and what gives a stream's handle.
PyObject *set_lm(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "set_lm(quantize, workspace, product, count, adjust, stream_of)");
        return nullptr;
    }
    void *at[5];
    for (int i = 0; i < 5; ++i)
        if (!(at[i] = PyLong_AsVoidPtr(args[i])) && PyErr_Occurred()) return nullptr;
    static_assert(sizeof(lm) == sizeof(at), "five functions");
    memcpy(&lm, at, sizeof(lm));
    Py_INCREF(args[5]);
    Py_XSETREF(stream_of, args[5]);
    Py_RETURN_NONE;
}

PyObject *set_general(PyObject *, PyObject *f) {
    Py_INCREF(f);
    Py_XSETREF(general, f);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"address", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(address)), METH_FASTCALL,
     "address(tensor, dtype, name): device address of a contiguous GPU tensor, 0 for None"},
    {"pack_jobs", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(pack_jobs)), METH_FASTCALL,
     "pack_jobs(rows, kinds, names): the bytes of an array of cnr_table_job"},
    {"batch_jobs", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(batch_jobs)), METH_FASTCALL,
     "batch_jobs(checkpointers, stage, tensors, outputs): the bytes of a batch's job array, or None where the general way has to look"},
    {"quantize_blocks", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(quantize_blocks)), METH_FASTCALL, "the call's status, or None"},
    {"block_product", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(block_product)), METH_FASTCALL, "the call's status, or None"},
    {"count_tokens", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(count_tokens)), METH_FASTCALL, "the call's status, or None"},
    {"adjust_logits", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(adjust_logits)), METH_FASTCALL, "the call's status, or None"},
    {"set_lm", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(set_lm)), METH_FASTCALL, "set_lm(quantize, workspace, product, count, adjust, stream_of): the library's functions"},
    {"set_general", set_general, METH_O, "set_general(f): what answers for tensors of other types"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() {
    for (int i = 0; i < kNameCount; ++i)
        if (!names[i] && !(names[i] = PyUnicode_InternFromString(kNames[i]))) return nullptr;
    if (!value_name && !(value_name = PyUnicode_InternFromString("value"))) return nullptr;
    return PyModule_Create(&module);
}
