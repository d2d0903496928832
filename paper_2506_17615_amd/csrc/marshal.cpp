// The binding's ordinary call, in native code: a torch tensor's checks, its pointer and the current stream are a few
// nanoseconds here and 0.2-0.3 us per tensor through the interpreter, where a call with 16 partial sums spent 11 us
// before its first launch (5 us with two; a launch itself takes the host 2.4 us).
//
// Every function takes the arguments of the Python function of its name, positionally, and returns the status of the C
// call it made, or -1 if it made none.  It makes the call only for arguments that the Python function would accept and
// hand on as they are: plain torch.Tensor objects on a GPU, of the expected type, contiguous and long enough, plain ints
// in range.  Everything else -- subclasses, wrappers without memory, anything to be refused -- is -1, and
// the caller goes through the checks in Python, which also word the errors.  Nothing is kept between calls.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "equarx.h"

namespace {

constexpr int kNotPlain = -1;
constexpr auto kBF16 = at::ScalarType::BFloat16;
constexpr auto kInt8 = at::ScalarType::Char;
constexpr auto kFloat = at::ScalarType::Float;
constexpr auto kByte = at::ScalarType::Byte;
constexpr auto kInt = at::ScalarType::Int;
constexpr auto kLong = at::ScalarType::Long;

// The library's entry points, as binding.load() found them.
struct Library {
#define EQUARX_CALLS(X)                                                                                              \
    X(equarx_quantize) X(equarx_quantize_batch) X(equarx_dequantize) X(equarx_reduce_stage) X(equarx_reduce_quantized) \
    X(equarx_reduce_quantized_static) X(equarx_reduce_quantized_fused_ends) X(equarx_reduce_fused)                   \
    X(equarx_reduce_variant) X(equarx_reduce_variant_hops) X(equarx_reduce_flat) X(equarx_quantize_strided)          \
    X(equarx_dequantize_strided) X(equarx_reduce_stage_strided) X(equarx_reduce_quantized_strided)                   \
    X(equarx_reduce_fused_strided) X(equarx_reduce_variant_strided) X(equarx_reduce_variant_hops_strided)            \
    X(equarx_mx4_quantize) X(equarx_mx4_dequantize) X(equarx_mx4_product) X(equarx_mx4_linear)                       \
    X(equarx_cache_write) X(equarx_cache_read) X(equarx_cache_attention)
#define X(name) decltype(&::name) name;
    EQUARX_CALLS(X)
#undef X
} lib;
bool bound = false;

// A tensor whose memory can be handed on as it is.
const at::Tensor *plain(PyObject *o)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.defined() && t.is_cuda() && t.has_storage() && t.is_contiguous() ? &t : nullptr;
}

struct Buffer {
    void *ptr = nullptr;
    int64_t count = 0;
    const at::Tensor *t = nullptr;

    bool of(PyObject *o, at::ScalarType type)
    {
        t = plain(o);
        if (!t || t->scalar_type() != type) return false;
        ptr = t->data_ptr();
        count = t->numel();
        return true;
    }
    bool of(PyObject *o, at::ScalarType type, int64_t at_least) { return of(o, type) && count >= at_least; }
};

// None, or any contiguous device tensor.
struct Workspace {
    void *ptr = nullptr;
    size_t bytes = 0;

    bool of(PyObject *o)
    {
        if (o == Py_None) return true;
        const at::Tensor *t = plain(o);
        if (!t) return false;
        ptr = t->data_ptr();
        bytes = (size_t)t->numel() * t->element_size();
        return true;
    }
};

bool integer(PyObject *o, long long lo, long long hi, long long &v)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return !overflow && v >= lo && v <= hi;
}

bool a_block(PyObject *o, int32_t &block)
{
    long long v;
    if (!integer(o, 32, 512, v) || (v & (v - 1))) return false;
    block = (int32_t)v;
    return true;
}

bool a_chunks(PyObject *o, int32_t &chunks) { return a_block(o, chunks) && chunks <= 128; }

bool some_flags(PyObject *o, uint32_t &flags)
{
    long long v;
    if (!integer(o, 0, UINT32_MAX, v)) return false;
    flags = (uint32_t)v;
    return true;
}

// A list or tuple of 1..EQUARX_MAX_PARTIALS tensors of one type, each of n elements (n < 0: the first one's length,
// which is then n) or, with `exactly` false, of at least n.
struct Buffers {
    void *ptr[EQUARX_MAX_PARTIALS];
    int32_t count = 0;

    bool of(PyObject *o, at::ScalarType type, int64_t &n, bool exactly = true)
    {
        if (!PyList_CheckExact(o) && !PyTuple_CheckExact(o)) return false;
        const Py_ssize_t size = PySequence_Fast_GET_SIZE(o);
        if (size < 1 || size > EQUARX_MAX_PARTIALS) return false;
        for (Py_ssize_t i = 0; i < size; ++i) {
            Buffer b;
            if (!b.of(PySequence_Fast_GET_ITEM(o, i), type)) return false;
            if (n < 0) n = b.count;
            if (exactly ? b.count != n : b.count < n) return false;
            ptr[i] = b.ptr;
        }
        count = (int32_t)size;
        return true;
    }
    template <typename T>
    T *const *as() const { return reinterpret_cast<T *const *>(ptr); }
    const void *const *partials() const { return ptr; }
};

void *stream() { return c10::hip::getCurrentHIPStream().stream(); }

int64_t blocks(int64_t n, int32_t block) { return (n + block - 1) / block; }
int64_t row(int64_t n, int64_t multiple) { return (n + multiple - 1) / multiple * multiple; }

template <typename F, typename... A>
int call(F f, A... args)
{
    void *const on = stream();      // may throw: not without the interpreter lock
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = f(args..., on);
    Py_END_ALLOW_THREADS
    return status;
}

// What every chain call starts with: partials, block (or chunks), and an output of their length.
struct Chain {
    Buffers x;
    int64_t n = -1;
    int32_t block = 0;
    Buffer out;

    bool of(PyObject *partials, PyObject *b, PyObject *o, bool strided = false)
    {
        return x.of(partials, kBF16, n) && n > 0 && (strided ? a_chunks(b, block) : a_block(b, block)) && out.of(o, kBF16, n);
    }
};

// The wire a chain call may keep: both arrays or neither.
struct KeptWire {
    Buffer codes, scales;

    bool of(PyObject *c, PyObject *s, const Chain &k)
    {
        if (c == Py_None && s == Py_None) return true;
        return codes.of(c, kInt8, k.x.count * row(k.n, 16)) && scales.of(s, kFloat, k.x.count * row(blocks(k.n, k.block), 4));
    }
};

int quantize(PyObject *const *a, bool strided)
{
    Buffer x, codes, scales;
    int32_t b;
    if (!x.of(a[0], kBF16) || x.count == 0 || !(strided ? a_chunks(a[1], b) : a_block(a[1], b))) return kNotPlain;
    if (!codes.of(a[2], kInt8, x.count)) return kNotPlain;
    if (!scales.of(a[3], kFloat, strided ? x.count / b : blocks(x.count, b))) return kNotPlain;
    return call(strided ? lib.equarx_quantize_strided : lib.equarx_quantize, x.ptr, x.count, b,
                static_cast<int8_t *>(codes.ptr), static_cast<float *>(scales.ptr));
}

int dequantize(PyObject *const *a, bool strided)
{
    Buffer codes, scales, out;
    int32_t b;
    if (!codes.of(a[0], kInt8) || codes.count == 0 || !(strided ? a_chunks(a[2], b) : a_block(a[2], b))) return kNotPlain;
    if (!scales.of(a[1], kFloat, strided ? codes.count / b : blocks(codes.count, b))) return kNotPlain;
    if (!out.of(a[3], kBF16, codes.count)) return kNotPlain;
    return call(strided ? lib.equarx_dequantize_strided : lib.equarx_dequantize, static_cast<const int8_t *>(codes.ptr),
                static_cast<const float *>(scales.ptr), codes.count, b, out.ptr);
}

int reduce_stage(PyObject *const *a, bool strided)
{
    Buffer cin, sin, local, cout, sout;
    int32_t b;
    if (!local.of(a[2], kBF16) || local.count == 0 || !(strided ? a_chunks(a[3], b) : a_block(a[3], b))) return kNotPlain;
    const int64_t n = local.count, ns = strided ? n / b : blocks(n, b);
    if (!cin.of(a[0], kInt8, n) || !cout.of(a[4], kInt8, n)) return kNotPlain;
    if (!sin.of(a[1], kFloat, ns) || !sout.of(a[5], kFloat, ns)) return kNotPlain;
    return call(strided ? lib.equarx_reduce_stage_strided : lib.equarx_reduce_stage, static_cast<const int8_t *>(cin.ptr),
                static_cast<const float *>(sin.ptr), local.ptr, n, b, static_cast<int8_t *>(cout.ptr),
                static_cast<float *>(sout.ptr));
}

int quantize_batch(PyObject *const *a)
{
    Buffers x, codes, scales;
    int64_t n = -1;
    int32_t block;
    if (!x.of(a[0], kBF16, n) || n == 0 || !a_block(a[1], block)) return kNotPlain;
    int64_t nb = blocks(n, block);
    if (!codes.of(a[2], kInt8, n, false) || !scales.of(a[3], kFloat, nb, false)) return kNotPlain;
    if (codes.count != x.count || scales.count != x.count) return kNotPlain;
    return call(lib.equarx_quantize_batch, x.partials(), codes.as<int8_t>(), scales.as<float>(), x.count, n, block);
}

int reduce_quantized(PyObject *const *a)
{
    Chain k;
    Workspace w;
    KeptWire wire;
    if (!k.of(a[0], a[1], a[2]) || !w.of(a[3]) || !wire.of(a[4], a[5], k)) return kNotPlain;
    return call(lib.equarx_reduce_quantized, k.x.partials(), k.x.count, k.n, k.block, k.out.ptr, w.ptr, w.bytes,
                static_cast<int8_t *>(wire.codes.ptr), static_cast<float *>(wire.scales.ptr));
}

int reduce_quantized_static(PyObject *const *a)
{
    Chain k;
    if (!k.of(a[0], a[1], a[2])) return kNotPlain;
    return call(lib.equarx_reduce_quantized_static, k.x.partials(), k.x.count, k.n, k.block, k.out.ptr);
}

int reduce_quantized_fused_ends(PyObject *const *a)
{
    Chain k;
    Workspace w;
    if (!k.of(a[0], a[1], a[2]) || !w.of(a[3])) return kNotPlain;
    return call(lib.equarx_reduce_quantized_fused_ends, k.x.partials(), k.x.count, k.n, k.block, k.out.ptr, w.ptr, w.bytes);
}

int reduce_fused(PyObject *const *a)
{
    Chain k;
    KeptWire wire;
    if (!k.of(a[0], a[1], a[2]) || !wire.of(a[3], a[4], k)) return kNotPlain;
    return call(lib.equarx_reduce_fused, k.x.partials(), k.x.count, k.n, k.block, k.out.ptr,
                static_cast<int8_t *>(wire.codes.ptr), static_cast<float *>(wire.scales.ptr));
}

int reduce_variant(PyObject *const *a, bool strided)
{
    Chain k;
    uint32_t flags;
    if (!k.of(a[0], a[1], a[3], strided) || !some_flags(a[2], flags)) return kNotPlain;
    return call(strided ? lib.equarx_reduce_variant_strided : lib.equarx_reduce_variant, k.x.partials(), k.x.count, k.n,
                k.block, flags, k.out.ptr);
}

int reduce_variant_hops(PyObject *const *a, bool strided)
{
    Chain k;
    uint32_t flags;
    Workspace w;
    if (!k.of(a[0], a[1], a[3], strided) || !some_flags(a[2], flags)) return kNotPlain;
    if ((strided && a[4] == Py_None) || !w.of(a[4])) return kNotPlain;
    return call(strided ? lib.equarx_reduce_variant_hops_strided : lib.equarx_reduce_variant_hops, k.x.partials(),
                k.x.count, k.n, k.block, flags, k.out.ptr, w.ptr, w.bytes);
}

int reduce_quantized_strided(PyObject *const *a)
{
    Chain k;
    Workspace w;
    if (!k.of(a[0], a[1], a[2], true) || !w.of(a[3])) return kNotPlain;
    return call(lib.equarx_reduce_quantized_strided, k.x.partials(), k.x.count, k.n, k.block, k.out.ptr, w.ptr, w.bytes);
}

int reduce_fused_strided(PyObject *const *a)
{
    Chain k;
    if (!k.of(a[0], a[1], a[2], true)) return kNotPlain;
    return call(lib.equarx_reduce_fused_strided, k.x.partials(), k.x.count, k.n, k.block, k.out.ptr);
}

int reduce_flat(PyObject *const *a)
{
    Buffer local, out, codes_out, scales_out;
    Buffers codes, scales;
    int32_t block;
    if (!local.of(a[0], kBF16) || local.count == 0 || !a_block(a[3], block)) return kNotPlain;
    int64_t n = local.count, nb = blocks(n, block);
    if (!codes.of(a[1], kInt8, n, false) || !scales.of(a[2], kFloat, nb, false)) return kNotPlain;
    if (codes.count != scales.count) return kNotPlain;
    if (a[4] != Py_None && !out.of(a[4], kBF16, n)) return kNotPlain;
    if (a[5] != Py_None || a[6] != Py_None) {
        if (!codes_out.of(a[5], kInt8, n) || !scales_out.of(a[6], kFloat, nb)) return kNotPlain;
    }
    return call(lib.equarx_reduce_flat, local.ptr, codes.as<const int8_t>(), scales.as<const float>(), codes.count, n, block,
                out.ptr, static_cast<int8_t *>(codes_out.ptr), static_cast<float *>(scales_out.ptr));
}

// ---------------------------------------------------------------- 4-bit rows and the cache

// A bf16 tensor of `dims` dimensions whose last one is contiguous; `row` and `head` are the strides of the first and (with
// three) the second, those of a packed tensor where there is but one index.
struct Rows {
    void *ptr = nullptr;
    int64_t size[3] = {0, 0, 0}, row = 0, head = 0;

    bool of(PyObject *o, int dims)
    {
        if (!THPVariable_CheckExact(o)) return false;
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.defined() || !t.is_cuda() || !t.has_storage() || t.scalar_type() != kBF16 || t.dim() != dims) return false;
        if (t.numel() == 0) return false;
        for (int i = 0; i < dims; ++i) size[i] = t.size(i);
        const int64_t cols = size[dims - 1];
        if (cols > 1 && t.stride(dims - 1) != 1) return false;
        head = dims == 3 && size[1] > 1 ? t.stride(1) : cols;
        row = size[0] > 1 ? t.stride(0) : dims == 3 ? size[1] * cols : cols;
        ptr = t.data_ptr();
        return true;
    }
};

// uint8 codes [rows][16 * blocks] and scales [rows][blocks], contiguous.
struct PackedRows {
    uint8_t *codes = nullptr, *scales = nullptr;
    int64_t rows = 0;

    bool of(PyObject *c, PyObject *s, int64_t cols)
    {
        const at::Tensor *tc = plain(c), *ts = plain(s);
        if (!tc || !ts || tc->scalar_type() != kByte || ts->scalar_type() != kByte || tc->dim() != 2 || ts->dim() != 2)
            return false;
        const int64_t per = (cols + EQUARX_MX4_GROUP - 1) / EQUARX_MX4_GROUP * (EQUARX_MX4_GROUP / EQUARX_MX4_BLOCK);
        rows = tc->size(0);
        if (ts->size(0) != rows || tc->size(1) != 16 * per || ts->size(1) != per) return false;
        codes = static_cast<uint8_t *>(tc->data_ptr());
        scales = static_cast<uint8_t *>(ts->data_ptr());
        return true;
    }
};

int mx4_quantize(PyObject *const *a)
{
    Rows x;
    PackedRows p;
    if (!x.of(a[0], 2) || !p.of(a[1], a[2], x.size[1]) || p.rows != x.size[0]) return kNotPlain;
    return call(lib.equarx_mx4_quantize, x.ptr, x.size[0], x.size[1], x.row, p.codes, p.scales);
}

int mx4_dequantize(PyObject *const *a)
{
    Rows out;
    PackedRows p;
    if (!out.of(a[2], 2) || !p.of(a[0], a[1], out.size[1]) || p.rows != out.size[0]) return kNotPlain;
    return call(lib.equarx_mx4_dequantize, p.codes, p.scales, out.size[0], out.size[1], out.ptr, out.row);
}

int mx4_product(PyObject *const *a)
{
    Rows out;
    PackedRows x, w;
    Workspace ws;
    long long K;
    if (!integer(a[4], 1, INT32_MAX, K) || !out.of(a[5], 2) || !x.of(a[0], a[1], K) || !w.of(a[2], a[3], K) || !ws.of(a[6]))
        return kNotPlain;
    if (x.rows != out.size[0] || w.rows != out.size[1]) return kNotPlain;
    return call(lib.equarx_mx4_product, x.codes, x.scales, w.codes, w.scales, out.size[0], out.size[1], (int64_t)K, out.ptr,
                out.row, ws.ptr, ws.bytes);
}

int mx4_linear(PyObject *const *a)
{
    Rows x, out;
    PackedRows w;
    Workspace ws;
    if (!x.of(a[0], 2) || !w.of(a[1], a[2], x.size[1]) || !out.of(a[3], 2) || !ws.of(a[4])) return kNotPlain;
    if (x.size[0] != out.size[0] || w.rows != out.size[1]) return kNotPlain;
    return call(lib.equarx_mx4_linear, x.ptr, x.row, w.codes, w.scales, out.size[0], out.size[1], x.size[1], out.ptr, out.row,
                ws.ptr, ws.bytes);
}

// A Cache: a tuple of four tensors of the shapes that the header gives.
bool a_cache(PyObject *o, equarx_cache &c)
{
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4) return false;
    const at::Tensor *t[4];
    for (int i = 0; i < 4; ++i) {
        t[i] = plain(PyTuple_GET_ITEM(o, i));
        if (!t[i] || t[i]->scalar_type() != (i % 2 ? kFloat : kInt8) || t[i]->dim() != (i == 2 ? 5 : 4) || t[i]->numel() == 0)
            return false;
    }
    const int64_t pages = t[0]->size(0), heads = t[0]->size(1), page = t[0]->size(2), dim = t[0]->size(3), blocks = t[1]->size(2);
    if (heads > INT32_MAX || page > INT32_MAX || dim > INT32_MAX || blocks < 1 || dim % blocks != 0) return false;
    for (int i = 1; i < 4; i += 2) {
        if (t[i]->size(0) != pages || t[i]->size(1) != heads || t[i]->size(2) != blocks || t[i]->size(3) != page) return false;
    }
    if (t[2]->size(0) != pages || t[2]->size(1) != heads || t[2]->size(2) * 16 != page || t[2]->size(3) != dim ||
        t[2]->size(4) != 16)
        return false;
    c.k_codes = static_cast<int8_t *>(t[0]->data_ptr());
    c.k_scales = static_cast<float *>(t[1]->data_ptr());
    c.v_codes = static_cast<int8_t *>(t[2]->data_ptr());
    c.v_scales = static_cast<float *>(t[3]->data_ptr());
    c.pages = pages;
    c.heads = (int32_t)heads;
    c.page = (int32_t)page;
    c.dim = (int32_t)dim;
    c.block = (int32_t)(dim / blocks);
    return true;
}

bool same_heads(const Rows &r, const equarx_cache &c) { return r.size[1] == c.heads && r.size[2] == c.dim; }

// page_table [sequences][width] and lengths [sequences].
struct SequenceList {
    const int32_t *table = nullptr, *lengths = nullptr;
    int64_t width = 0;
    int32_t count = 0;

    bool of(PyObject *tab, PyObject *len)
    {
        Buffer t, n;
        if (!t.of(tab, kInt) || t.t->dim() != 2 || t.count == 0 || t.t->size(0) > INT32_MAX) return false;
        count = (int32_t)t.t->size(0);
        width = t.t->size(1);
        if (!n.of(len, kInt) || n.count != count) return false;
        table = static_cast<const int32_t *>(t.ptr);
        lengths = static_cast<const int32_t *>(n.ptr);
        return true;
    }
};

int cache_write(PyObject *const *a)
{
    equarx_cache c;
    Rows k, v;
    Buffer slots;
    if (!a_cache(a[0], c) || !k.of(a[1], 3) || !v.of(a[2], 3) || !same_heads(k, c) || !same_heads(v, c)) return kNotPlain;
    if (v.size[0] != k.size[0] || !slots.of(a[3], kLong) || slots.count != k.size[0]) return kNotPlain;
    return call(lib.equarx_cache_write, &c, k.ptr, k.row, k.head, v.ptr, v.row, v.head, k.size[0],
                static_cast<const int64_t *>(slots.ptr));
}

int cache_read(PyObject *const *a)
{
    equarx_cache c;
    SequenceList seqs;
    Buffer starts;
    long long longest;
    if (!a_cache(a[0], c) || !seqs.of(a[1], a[2]) || !starts.of(a[3], kInt, seqs.count)) return kNotPlain;
    const at::Tensor *const k = plain(a[4]), *const v = plain(a[5]);
    for (const at::Tensor *t : {k, v}) {
        if (!t || t->scalar_type() != kBF16 || t->dim() != 3 || t->numel() == 0 || t->size(1) != c.heads || t->size(2) != c.dim)
            return kNotPlain;
    }
    if (k->size(0) != v->size(0) || !integer(a[6], 0, INT64_MAX, longest)) return kNotPlain;
    return call(lib.equarx_cache_read, &c, seqs.table, seqs.width, seqs.lengths, static_cast<const int32_t *>(starts.ptr),
                seqs.count, (int64_t)longest, k->size(0), k->data_ptr(), v->data_ptr());
}

int cache_attention(PyObject *const *a)
{
    equarx_cache c;
    Rows q;
    SequenceList seqs;
    Buffer starts, out, lse;
    Workspace ws;
    long long queries, longest, window;
    if (!a_cache(a[0], c) || !q.of(a[1], 3) || q.size[2] != c.dim || q.size[1] > INT32_MAX || !seqs.of(a[3], a[4])) return kNotPlain;
    if (!starts.of(a[2], kInt) || starts.count != (int64_t)seqs.count + 1) return kNotPlain;
    if (!out.of(a[5], kBF16) || out.t->dim() != 3 || out.t->size(0) != q.size[0] || out.t->size(1) != q.size[1] ||
        out.t->size(2) != q.size[2])
        return kNotPlain;
    if (!PyFloat_CheckExact(a[6]) || !integer(a[7], 1, INT32_MAX, queries) || !integer(a[8], 1, INT32_MAX, longest)) return kNotPlain;
    if (!PyBool_Check(a[9]) || !integer(a[10], 0, INT32_MAX, window)) return kNotPlain;
    if (a[11] != Py_None && (!lse.of(a[11], kFloat) || lse.count != q.size[0] * q.size[1])) return kNotPlain;
    if (!ws.of(a[12])) return kNotPlain;
    return call(lib.equarx_cache_attention, &c, q.ptr, q.size[0], (int32_t)q.size[1], q.row, q.head,
                static_cast<const int32_t *>(starts.ptr), seqs.table, seqs.width, seqs.lengths, seqs.count,
                (float)PyFloat_AS_DOUBLE(a[6]), (int32_t)queries, (int64_t)longest,
                a[9] == Py_True ? EQUARX_CAUSAL : 0u, (int32_t)window, out.ptr, static_cast<float *>(lse.ptr), ws.ptr, ws.bytes);
}

// The Python-callable form of f: kArgs positional arguments; an exception from torch is "not plain" too.
template <int kArgs, typename F>
PyObject *enter(PyObject *const *a, Py_ssize_t count, F f)
{
    int status = kNotPlain;
    if (!bound) {
        PyErr_SetString(PyExc_RuntimeError, "not bound to a library");
        return nullptr;
    }
    if (count == kArgs) {
        try {
            status = f(a);
        } catch (...) {
            status = kNotPlain;
        }
    }
    return PyLong_FromLong(status);
}

#define ENTRY(args, name, expr)                                                       \
    PyObject *py_##name(PyObject *, PyObject *const *a, Py_ssize_t count)             \
    {                                                                                 \
        return enter<args>(a, count, [](PyObject *const *a) { return expr; });        \
    }
ENTRY(4, equarx_quantize, quantize(a, false))
ENTRY(4, equarx_quantize_batch, quantize_batch(a))
ENTRY(4, equarx_dequantize, dequantize(a, false))
ENTRY(6, equarx_reduce_stage, reduce_stage(a, false))
ENTRY(6, equarx_reduce_quantized, reduce_quantized(a))
ENTRY(3, equarx_reduce_quantized_static, reduce_quantized_static(a))
ENTRY(4, equarx_reduce_quantized_fused_ends, reduce_quantized_fused_ends(a))
ENTRY(5, equarx_reduce_fused, reduce_fused(a))
ENTRY(4, equarx_reduce_variant, reduce_variant(a, false))
ENTRY(5, equarx_reduce_variant_hops, reduce_variant_hops(a, false))
ENTRY(7, equarx_reduce_flat, reduce_flat(a))
ENTRY(4, equarx_quantize_strided, quantize(a, true))
ENTRY(4, equarx_dequantize_strided, dequantize(a, true))
ENTRY(6, equarx_reduce_stage_strided, reduce_stage(a, true))
ENTRY(4, equarx_reduce_quantized_strided, reduce_quantized_strided(a))
ENTRY(3, equarx_reduce_fused_strided, reduce_fused_strided(a))
ENTRY(4, equarx_reduce_variant_strided, reduce_variant(a, true))
ENTRY(5, equarx_reduce_variant_hops_strided, reduce_variant_hops(a, true))
ENTRY(3, equarx_mx4_quantize, mx4_quantize(a))
ENTRY(3, equarx_mx4_dequantize, mx4_dequantize(a))
ENTRY(7, equarx_mx4_product, mx4_product(a))
ENTRY(5, equarx_mx4_linear, mx4_linear(a))
ENTRY(4, equarx_cache_write, cache_write(a))
ENTRY(7, equarx_cache_read, cache_read(a))
ENTRY(13, equarx_cache_attention, cache_attention(a))
#undef ENTRY

// bind({name: address}): where the library's entry points are.
PyObject *bind(PyObject *, PyObject *table)
{
    Library found;
#define X(name)                                                                       \
    {                                                                                 \
        PyObject *at = PyDict_Check(table) ? PyDict_GetItemString(table, #name) : nullptr; \
        void *p = at ? PyLong_AsVoidPtr(at) : nullptr;                                \
        if (!p) {                                                                     \
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no address for " #name); \
            return nullptr;                                                           \
        }                                                                             \
        found.name = reinterpret_cast<decltype(&::name)>(p);                          \
    }
    EQUARX_CALLS(X)
#undef X
    lib = found;
    bound = true;
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
#define X(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(py_##name)), METH_FASTCALL, nullptr},
    EQUARX_CALLS(X)
#undef X
    {"bind", bind, METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal()
{
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "torch_version", EQUARX_TORCH) < 0) Py_CLEAR(m);
    return m;
}
