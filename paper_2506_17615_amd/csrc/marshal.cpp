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
#include <c10/hip/HIPFunctions.h>
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
    X(equarx_cache_write) X(equarx_cache_read) X(equarx_cache_attention)                                             \
    X(equarx_norm) X(equarx_norm_reduced) X(equarx_pages_trim) X(equarx_pages_extend) X(equarx_adapters)
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
    const at::Tensor *tensor = nullptr;

    bool of(PyObject *o, int dims)
    {
        if (!THPVariable_CheckExact(o)) return false;
        const at::Tensor &t = THPVariable_Unpack(o);
        tensor = &t;
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

// ---------------------------------------------------------------- norms

// On the device whose stream the call is made on?  A call that asks sets it first.
thread_local c10::DeviceIndex current_device = -1;

bool here(const at::Tensor *t) { return !t || t->device().index() == current_device; }

// The arguments of a norm of [rows][cols] from `weight` on: weight, eps, residual, out, codes, scales, their block, packed codes and
// scales, whether 1 is added to the weight.
struct Norm {
    Buffer weight, codes, scales;
    Rows residual, out;
    PackedRows packed;
    double eps = 0;
    uint32_t flags = 0;
    equarx_norm_outputs to{};

    bool of(PyObject *const *a, int64_t rows, int64_t cols)
    {
        auto sized = [&](const Rows &r) { return r.size[0] == rows && r.size[1] == cols && here(r.tensor); };
        if (a[0] != Py_None && (!weight.of(a[0], kBF16) || weight.count != cols || !here(weight.t))) return false;
        if (!PyFloat_CheckExact(a[1]) || !PyBool_Check(a[9])) return false;
        eps = PyFloat_AS_DOUBLE(a[1]);
        flags = a[9] == Py_True ? EQUARX_NORM_ONE_PLUS : 0u;
        if (a[2] != Py_None && (!residual.of(a[2], 2) || !sized(residual))) return false;
        if (a[3] != Py_None && (!out.of(a[3], 2) || !sized(out))) return false;
        if (a[4] != Py_None || a[5] != Py_None) {
            if (!a_block(a[6], to.block) || !codes.of(a[4], kInt8, rows * cols) || !here(codes.t)) return false;
            if (!scales.of(a[5], kFloat, blocks(rows * cols, to.block)) || !here(scales.t)) return false;
        } else {
            long long unused;
            if (!integer(a[6], 0, INT32_MAX, unused)) return false;
        }
        if (a[7] != Py_None || a[8] != Py_None) {
            if (!packed.of(a[7], a[8], cols) || packed.rows != rows || !here(plain(a[7])) || !here(plain(a[8]))) return false;
        }
        to.out_bf16 = out.ptr;
        to.out_stride = out.row;
        to.codes = static_cast<int8_t *>(codes.ptr);
        to.scales = static_cast<float *>(scales.ptr);
        to.mx4_codes = packed.codes;
        to.mx4_scales = packed.scales;
        return true;
    }
};

int norm(PyObject *const *a)
{
    current_device = c10::hip::current_device();
    Rows x;
    Norm n;
    if (!x.of(a[0], 2) || !here(x.tensor) || !n.of(a + 1, x.size[0], x.size[1])) return kNotPlain;
    return call(lib.equarx_norm, x.ptr, x.row, n.residual.ptr, n.residual.row, n.weight.ptr, x.size[0], x.size[1], n.eps, n.flags, &n.to);
}

int norm_reduced(PyObject *const *a)
{
    current_device = c10::hip::current_device();
    Buffers x;
    Norm n;
    int64_t count = -1;
    int32_t block;
    if (!x.of(a[0], kBF16, count) || count == 0 || !a_block(a[1], block)) return kNotPlain;
    int64_t rows = 0, cols = 0;
    for (int32_t i = 0; i < x.count; ++i) {
        const at::Tensor &t = THPVariable_Unpack(PySequence_Fast_GET_ITEM(a[0], i));
        if (t.dim() != 2 || !here(&t) || (i > 0 && (t.size(0) != rows || t.size(1) != cols))) return kNotPlain;
        rows = t.size(0);
        cols = t.size(1);
    }
    if (!n.of(a + 2, rows, cols)) return kNotPlain;
    return call(lib.equarx_norm_reduced, x.partials(), x.count, block, n.residual.ptr, n.residual.row, n.weight.ptr, rows, cols, n.eps,
                n.flags, &n.to);
}

// ---------------------------------------------------------------- pages and adapters

// A contiguous tensor of the current device with exactly `count` elements.
bool exactly(Buffer &b, PyObject *o, at::ScalarType type, int64_t count) { return b.of(o, type) && b.count == count && here(b.t); }

// A Pages (a tuple of four tensors) and the tokens of a page.
bool some_pages(PyObject *o, PyObject *page, equarx_pages &p)
{
    long long size;
    Buffer table, lengths, free, count;
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 4 || !integer(page, 1, 65536, size)) return false;
    if (!table.of(PyTuple_GET_ITEM(o, 0), kInt) || table.t->dim() != 2 || table.count == 0 || table.t->size(0) > INT32_MAX || !here(table.t))
        return false;
    p.sequences = (int32_t)table.t->size(0);
    p.width = table.t->size(1);
    if (!exactly(lengths, PyTuple_GET_ITEM(o, 1), kInt, p.sequences) || !exactly(count, PyTuple_GET_ITEM(o, 3), kInt, 1)) return false;
    if (!free.of(PyTuple_GET_ITEM(o, 2), kInt) || free.t->dim() != 1 || !here(free.t)) return false;
    p.table = static_cast<int32_t *>(table.ptr);
    p.lengths = static_cast<int32_t *>(lengths.ptr);
    p.free = static_cast<int32_t *>(free.ptr);
    p.free_count = static_cast<int32_t *>(count.ptr);
    p.pages = free.count;
    p.page = (int32_t)size;
    p.seen = nullptr;
    return true;
}

int pages_trim(PyObject *const *a)
{
    current_device = c10::hip::current_device();
    equarx_pages p;
    Buffer keep;
    if (!some_pages(a[0], a[1], p) || !exactly(keep, a[2], kInt, p.sequences)) return kNotPlain;
    return call(lib.equarx_pages_trim, &p, static_cast<const int32_t *>(keep.ptr));
}

// With `seen`, or without that argument.
int pages_extend(PyObject *const *a, bool with_seen)
{
    current_device = c10::hip::current_device();
    equarx_pages p;
    Buffer counts, starts, slots, granted, positions, tags, row_tags, seen;
    if (!some_pages(a[0], a[1], p) || !exactly(counts, a[2], kInt, p.sequences) || !exactly(starts, a[3], kInt, (int64_t)p.sequences + 1))
        return kNotPlain;
    if (!slots.of(a[4], kLong) || !here(slots.t)) return kNotPlain;
    if (a[5] != Py_None && !exactly(granted, a[5], kInt, p.sequences)) return kNotPlain;
    if (a[6] != Py_None && !exactly(positions, a[6], kInt, slots.count)) return kNotPlain;
    if (a[7] != Py_None && !exactly(tags, a[7], kInt, p.sequences)) return kNotPlain;
    if (a[8] != Py_None && !exactly(row_tags, a[8], kInt, slots.count)) return kNotPlain;
    if (with_seen && a[9] != Py_None && !exactly(seen, a[9], kInt, p.sequences)) return kNotPlain;
    p.seen = static_cast<int32_t *>(seen.ptr);
    return call(lib.equarx_pages_extend, &p, static_cast<const int32_t *>(counts.ptr), static_cast<int32_t *>(starts.ptr),
                static_cast<int64_t *>(slots.ptr), static_cast<int32_t *>(granted.ptr), static_cast<int32_t *>(positions.ptr),
                static_cast<const int32_t *>(tags.ptr), static_cast<int32_t *>(row_tags.ptr), slots.count);
}

int adapters(PyObject *const *a)
{
    current_device = c10::hip::current_device();
    Rows x, out;
    Buffer da, db, factors, ids;
    Workspace ws;
    int64_t ends[EQUARX_ADAPTERS_MAX_SLICES];
    Py_ssize_t slices = 1;
    if (!x.of(a[0], 2) || !here(x.tensor) || !out.of(a[5], 2) || !here(out.tensor) || out.size[0] != x.size[0]) return kNotPlain;
    const int64_t M = x.size[0], K = x.size[1], N = out.size[1];
    if (a[6] == Py_None) {
        ends[0] = N;
    } else {
        if (!PyTuple_CheckExact(a[6])) return kNotPlain;
        slices = PyTuple_GET_SIZE(a[6]);
        if (slices < 1 || slices > EQUARX_ADAPTERS_MAX_SLICES) return kNotPlain;
        for (Py_ssize_t i = 0; i < slices; ++i) {
            long long end;
            if (!integer(PyTuple_GET_ITEM(a[6], i), 0, INT32_MAX, end)) return kNotPlain;
            ends[i] = end;
        }
    }
    if (!da.of(a[1], kBF16) || da.t->dim() != 3 || !here(da.t) || !db.of(a[2], kBF16) || db.t->dim() != 3 || !here(db.t)) return kNotPlain;
    const int64_t count = db.t->size(0), rank = db.t->size(2);
    if (count > INT32_MAX || rank > INT32_MAX || db.t->size(1) != N || da.t->size(0) != count || da.t->size(1) != slices * rank ||
        da.t->size(2) != K)
        return kNotPlain;
    if (!exactly(factors, a[3], kFloat, count) || !exactly(ids, a[4], kInt, M) || !ws.of(a[7])) return kNotPlain;
    if (a[7] != Py_None && !here(plain(a[7]))) return kNotPlain;
    return call(lib.equarx_adapters, x.ptr, x.row, da.ptr, db.ptr, static_cast<const float *>(factors.ptr), (int32_t)count, (int32_t)rank,
                static_cast<const int32_t *>(ids.ptr), M, N, K, static_cast<const int64_t *>(ends), (int32_t)slices, out.ptr, out.row, ws.ptr,
                ws.bytes);
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
ENTRY(11, equarx_norm, norm(a))
ENTRY(12, equarx_norm_reduced, norm_reduced(a))
ENTRY(3, equarx_pages_trim, pages_trim(a))
ENTRY(8, equarx_adapters, adapters(a))
#undef ENTRY
PyObject *py_equarx_pages_extend(PyObject *, PyObject *const *a, Py_ssize_t count)
{
    if (count == 10) return enter<10>(a, count, [](PyObject *const *a) { return pages_extend(a, true); });
    return enter<9>(a, count, [](PyObject *const *a) { return pages_extend(a, false); });
}

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
