// Native argument marshalling for the entry points that a decode step calls with a dozen tensors each: page tables, the 4-bit
// cache, rules on logits.  It reads types, layouts, devices and addresses out of the tensors directly and calls the C ABI
// (include/psa.h), so that a call costs about as much as its launch; the same checks made attribute by attribute in Python
// took 6 to 11 us a call.  No arithmetic happens here, and the only memory is what a call on an explicit stream needs.
//
// What a caller got wrong about its tensors (type, layout, size, device) is raised as ValueError; the library's own status comes back as
// an integer, which the Python side turns into PsaError.
#include <Python.h>

#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <dlfcn.h>

#include <algorithm>
#include <stdexcept>
#include <string>

#include "psa.h"

namespace {

struct Refused : std::runtime_error {
    using std::runtime_error::runtime_error;
};

struct Api {
    decltype(&psa_build_page_table) build_page_table;
    decltype(&psa_extend_page_table) extend_page_table;
    decltype(&psa_store_kv4) store_kv4;
    decltype(&psa_load_kv4) load_kv4;
    decltype(&psa_decode_kv4) decode_kv4;
    decltype(&psa_process_logits) process_logits;
    decltype(&psa_mark_tokens) mark_tokens;
} api{};

const char *name_of(at::ScalarType t)
{
    switch (t) {
        case at::kInt: return "torch.int32";
        case at::kLong: return "torch.int64";
        case at::kByte: return "torch.uint8";
        case at::kBFloat16: return "torch.bfloat16";
        case at::kFloat: return "torch.float32";
        default: return c10::toString(t);
    }
}

// The tensors of one call.  Every check but the devices' is made as a tensor is read; devices come last, in stream().
class Call {
public:
    Call(PyObject *const *args, Py_ssize_t given, Py_ssize_t wanted) : args_(args)
    {
        if (given != wanted) throw Refused("wrong number of arguments");
    }
    bool none(int i) const { return args_[i] == Py_None; }
    const at::Tensor &tensor(int i, const char *name)
    {
        if (!THPVariable_Check(args_[i])) throw Refused(std::string(name) + " must be a tensor");
        const at::Tensor &t = THPVariable_Unpack(args_[i]);
        const int device = t.is_cuda() ? t.get_device() : -1;
        if (device_ == kUnset) device_ = device;
        if (!odd_ && (device < 0 || device != device_)) odd_ = name;
        return t;
    }
    // address of a contiguous tensor of at least `size` elements; null for None
    template <class T = void>
    T *flat(int i, at::ScalarType type, const char *name, int64_t size = 0)
    {
        if (none(i)) return nullptr;
        const at::Tensor &t = tensor(i, name);
        if (t.scalar_type() != type) throw Refused(std::string(name) + " must be " + name_of(type) + ", not " + name_of(t.scalar_type()));
        if (!t.is_contiguous() || t.numel() < size)
            throw Refused(std::string(name) + " must be contiguous and hold at least " + std::to_string(size) + " elements");
        return static_cast<T *>(t.data_ptr());
    }
    template <class T = void>
    T *needed(int i, at::ScalarType type, const char *name, int64_t size = 0)
    {
        if (none(i)) throw Refused(std::string(name) + " is missing");
        return flat<T>(i, type, name, size);
    }
    int64_t numel(int i) const { return THPVariable_Unpack(args_[i]).numel(); }   // of a tensor read before
    int64_t integer(int i) const
    {
        const long long v = PyLong_AsLongLong(args_[i]);
        if (v == -1 && PyErr_Occurred()) throw Refused("");
        return v;
    }
    // a status word: an int32 tensor, or the workspace of a plan (uint8), whose first word it is; the library checks its alignment
    int32_t *status(int i)
    {
        if (none(i)) return nullptr;
        const at::Tensor &t = tensor(i, "status");
        if (t.scalar_type() == at::kByte) return flat<int32_t>(i, at::kByte, "status", 4);
        return flat<int32_t>(i, at::kInt, "status", 1);
    }
    // the stream of the call (None: torch's current one), once all tensors have been read: they have to live on the current device
    void *stream(int i)
    {
        if (odd_) throw Refused(std::string(odd_) + " must be on the current CUDA device");
        if (device_ != c10::cuda::current_device()) throw Refused("the tensors must be on the current CUDA device");
        if (none(i)) return c10::cuda::getCurrentCUDAStream(c10::DeviceIndex(device_)).stream();
        return handle(args_[i]);
    }
    // a stream given as its handle or as an object that has one
    static void *handle(PyObject *stream)
    {
        PyObject *h = PyLong_Check(stream) ? Py_NewRef(stream) : PyObject_GetAttrString(stream, "cuda_stream");
        if (!h) throw Refused("");
        void *p = PyLong_AsVoidPtr(h);
        Py_DECREF(h);
        if (!p && PyErr_Occurred()) throw Refused("");
        return p;
    }

private:
    static constexpr int kUnset = -2;
    PyObject *const *args_;
    int device_ = kUnset;
    const char *odd_ = nullptr;   // the first tensor that is not where the first one is, or not on a GPU
};

// Strides of dimensions 0 and 1 of a 3-d tensor whose last dimension is contiguous; a dimension of one element has none of its own.
void outer_strides(const at::Tensor &t, int64_t inner, const char *name, int64_t (&s)[2])
{
    if (t.dim() != 3 || t.size(2) != inner || (t.stride(2) != 1 && inner > 1))
        throw Refused(std::string(name) + " must be [.., .., " + std::to_string(inner) + "] with a contiguous last dimension");
    s[1] = t.size(1) > 1 ? t.stride(1) : inner;
    s[0] = t.size(0) > 1 ? t.stride(0) : std::max<int64_t>(1, t.size(1)) * std::max(s[1], inner);
}

template <class Body>
PyObject *guarded(Body body)
{
    try {
        return body();
    } catch (const Refused &e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, e.what());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown error while reading the tensors of a call");
    }
    return nullptr;
}
template <psa_status_t (*body)(PyObject *const *, Py_ssize_t)>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] { return PyLong_FromLong(body(args, n)); });
}

// seq_lens, reserve_lens, free_pages, free_count, free_count_out, page_indptr, page_indices, token_indptr, slot_map, lens_out, status,
// scratch, stream
psa_status_t build_page_table(PyObject *const *args, Py_ssize_t given)
{
    Call c(args, given, 13);
    const auto *seq = c.needed<int32_t>(0, at::kInt, "seq_lens");
    const int64_t n = c.numel(0);
    const auto *reserve = c.flat<int32_t>(1, at::kInt, "reserve_lens", n);
    const auto *free_pages = c.needed<int32_t>(2, at::kInt, "free_pages");
    auto *count = c.needed<int32_t>(3, at::kInt, "free_count", 1);
    auto *count_out = c.flat<int32_t>(4, at::kInt, "free_count_out", 1);
    auto *indptr = c.needed<int32_t>(5, at::kInt, "page_indptr", n + 1);
    auto *indices = c.needed<int32_t>(6, at::kInt, "page_indices");
    auto *tokens = c.needed<int32_t>(7, at::kInt, "token_indptr", n + 1);
    auto *slots = c.needed<int64_t>(8, at::kLong, "slot_map");
    auto *lens = c.flat<int32_t>(9, at::kInt, "lens_out", n);
    int32_t *status = c.status(10);
    void *scratch = c.needed(11, at::kByte, "scratch");
    void *stream = c.stream(12);
    if (n > 0x7fffffff) throw Refused("too many samples");
    return api.build_page_table(seq, reserve, int32_t(n), free_pages, count, count_out ? count_out : count, indptr, indices, c.numel(6), tokens, slots,
                                c.numel(8), lens, status, scratch, size_t(c.numel(11)), stream);
}

// held_lens, new_lens, max_lens, free_pages, free_count, free_count_out, page_indptr, page_indices, token_indptr, slot_map, lens_out, status,
// scratch, stream
psa_status_t extend_page_table(PyObject *const *args, Py_ssize_t given)
{
    Call c(args, given, 14);
    const auto *held = c.needed<int32_t>(0, at::kInt, "held_lens");
    const int64_t n = c.numel(0);
    const auto *fresh = c.needed<int32_t>(1, at::kInt, "new_lens", n);
    const auto *most = c.flat<int32_t>(2, at::kInt, "max_lens", n);
    const auto *free_pages = c.needed<int32_t>(3, at::kInt, "free_pages");
    auto *count = c.needed<int32_t>(4, at::kInt, "free_count", 1);
    auto *count_out = c.flat<int32_t>(5, at::kInt, "free_count_out", 1);
    const auto *indptr = c.needed<int32_t>(6, at::kInt, "page_indptr", n + 1);
    auto *indices = c.needed<int32_t>(7, at::kInt, "page_indices");
    auto *tokens = c.needed<int32_t>(8, at::kInt, "token_indptr", n + 1);
    auto *slots = c.needed<int64_t>(9, at::kLong, "slot_map");
    auto *lens = c.flat<int32_t>(10, at::kInt, "lens_out", n);
    int32_t *status = c.status(11);
    void *scratch = c.needed(12, at::kByte, "scratch");
    void *stream = c.stream(13);
    if (n > 0x7fffffff) throw Refused("too many samples");
    return api.extend_page_table(held, fresh, most, int32_t(n), free_pages, count, count_out ? count_out : count, indptr, indices, c.numel(7), tokens,
                                 slots, c.numel(9), lens, status, scratch, size_t(c.numel(12)), stream);
}

// K, V, slot_map, pool, status, stream: bf16 rows [T, Hkv, D] and a pool [pages, Hkv, 20 D] uint8
struct Kv4Call {
    const at::Tensor *k, *v, *pool;
    const int64_t *slots;
    int64_t tokens, kv_strides[2], pool_strides[2];
    int32_t heads, dim;
    int32_t *status;
    void *stream;
    Kv4Call(PyObject *const *args, Py_ssize_t given, const char *names)
    {
        Call c(args, given, 6);
        k = &c.tensor(0, names);
        v = &c.tensor(1, names);
        if (k->dim() != 3 || k->scalar_type() != at::kBFloat16 || v->scalar_type() != at::kBFloat16 || k->sizes() != v->sizes())
            throw Refused(std::string(names) + " must be bf16 [tokens, heads, head_dim] of the same shape and strides");
        tokens = k->size(0);
        if (k->size(1) > 0x7fffffff || k->size(2) > 0xffff) throw Refused(std::string(names) + " are too large");
        heads = int32_t(k->size(1));
        dim = int32_t(k->size(2));
        slots = c.needed<int64_t>(2, at::kLong, "slot_map", tokens);
        pool = &c.tensor(3, "pool");
        if (pool->scalar_type() != at::kByte || pool->dim() != 3 || pool->size(1) != heads)
            throw Refused("pool must be uint8 [pages, heads, kv4_cell_bytes(head_dim)]");
        int64_t v_strides[2];
        outer_strides(*k, dim, names, kv_strides);
        outer_strides(*v, dim, names, v_strides);
        if (tokens > 0 && (kv_strides[0] != v_strides[0] || kv_strides[1] != v_strides[1])) throw Refused(std::string(names) + " must have the same strides");
        outer_strides(*pool, 20 * dim, "pool", pool_strides);
        status = c.status(4);
        stream = c.stream(5);
    }
};
psa_status_t store_kv4(PyObject *const *args, Py_ssize_t given)
{
    const Kv4Call c(args, given, "new_k and new_v");
    return api.store_kv4(c.k->data_ptr(), c.v->data_ptr(), c.kv_strides, c.slots, c.tokens, c.heads, c.dim, c.pool->data_ptr(), c.pool_strides,
                         c.pool->size(0), c.status, c.stream);
}
psa_status_t load_kv4(PyObject *const *args, Py_ssize_t given)
{
    const Kv4Call c(args, given, "out_k and out_v");
    return api.load_kv4(c.pool->data_ptr(), c.pool_strides, c.pool->size(0), c.slots, c.tokens, c.heads, c.dim, c.k->data_ptr(), c.v->data_ptr(),
                        c.kv_strides, c.status, c.stream);
}

// The shared prefix, bf16: K and V with the same token and head stride (elements), `tokens` rows of `heads` x `dim` of each inside its storage.
struct Prefix {
    const void *k = nullptr, *v = nullptr;
    int64_t strides[2];
    // tensors at `at` and `at` + 1, strides behind them (None: the tensors' own where they are [tokens, heads, dim], else contiguous)
    Prefix(Call &c, int at, int64_t tokens, int64_t heads, int64_t dim)
    {
        const bool own = c.none(at + 2);
        strides[0] = own ? heads * dim : c.integer(at + 2);
        strides[1] = own ? dim : c.integer(at + 3);
        const at::Tensor *first = nullptr;
        for (int i = 0; i < 2; ++i) {
            if (c.none(at + i)) continue;
            const char *name = i ? "prefix_v" : "prefix_k";
            const at::Tensor &t = c.tensor(at + i, name);
            if (t.scalar_type() != at::kBFloat16) throw Refused("prefix_k and prefix_v must be torch.bfloat16");
            (i ? v : k) = t.data_ptr();
            if (tokens == 0) continue;   // nothing is read
            if (own) {
                int64_t mine[2] = {heads * dim, dim};
                if (t.dim() == 3 && t.size(1) == heads && t.size(2) == dim) outer_strides(t, dim, name, mine);
                else if (!t.is_contiguous()) throw Refused(std::string(name) + " must be [tokens, heads, head_dim] or contiguous, unless prefix_strides are given");
                if (t.numel() < tokens * heads * dim) throw Refused(std::string(name) + " must hold at least " + std::to_string(tokens) + " tokens");
                if (first && (mine[0] != strides[0] || mine[1] != strides[1])) throw Refused("prefix_k and prefix_v must have the same strides");
                strides[0] = mine[0]; strides[1] = mine[1];
                first = &t;
            }
            const __int128 last = __int128(tokens - 1) * strides[0] + __int128(heads - 1) * strides[1] + dim;   // the library refuses strides below 1
            if (last > int64_t(t.storage().nbytes() / 2) - t.storage_offset())
                throw Refused(std::string(name) + " must hold at least " + std::to_string(tokens) + " tokens at these strides");
        }
    }
};

// tokens of the packed prefix, KV heads, head dim, prefix_k, prefix_v, prefix stride 0, prefix stride 1, stream: the strides that decode_kv4 would use
PyObject *prefix_strides(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&] {
        Call c(args, n, 8);
        const Prefix prefix(c, 3, c.integer(0), c.integer(1), c.integer(2));
        if (!c.none(3) || !c.none(4)) c.stream(7);
        return Py_BuildValue("LL", static_cast<long long>(prefix.strides[0]), static_cast<long long>(prefix.strides[1]));
    });
}

// plan handle, samples, query heads, KV heads, head dim, f32 output?, tokens of the packed prefix, q, prefix_k, prefix_v, prefix stride 0,
// prefix stride 1, pool, page_indptr, page_indices, suffix_lens, out, lse, workspace, stream
psa_status_t decode_kv4(PyObject *const *args, Py_ssize_t given)
{
    Call c(args, given, 20);
    const auto *plan = reinterpret_cast<const psa_plan_t *>(PyLong_AsVoidPtr(args[0]));
    const int64_t rows = c.integer(1), heads = c.integer(2), kv = c.integer(3), dim = c.integer(4);
    const at::Tensor &pool = c.tensor(12, "pool");
    if (pool.scalar_type() != at::kByte || pool.dim() != 3 || pool.size(1) != kv)
        throw Refused("pool must be uint8 [pages, num_kv_heads, kv4_cell_bytes(head_dim)]");
    int64_t pool_strides[2];
    outer_strides(pool, 20 * dim, "pool", pool_strides);
    const void *q = c.needed(7, at::kBFloat16, "q", rows * heads * dim);
    const Prefix prefix(c, 8, c.integer(6), kv, dim);
    const auto *indptr = c.needed<int32_t>(13, at::kInt, "page_indptr", rows + 1);
    const auto *indices = c.needed<int32_t>(14, at::kInt, "page_indices");
    const auto *lens = c.needed<int32_t>(15, at::kInt, "suffix_lens", rows);
    void *out = c.needed(16, c.integer(5) ? at::kFloat : at::kBFloat16, "out", rows * heads * dim);
    auto *lse = c.needed<float>(17, at::kFloat, "lse", rows * heads);
    void *workspace = c.needed(18, at::kByte, "workspace");
    void *stream = c.stream(19);
    return api.decode_kv4(plan, q, prefix.k, prefix.v, prefix.strides, pool.data_ptr(), pool_strides, indptr, indices, lens, out, lse, workspace,
                          size_t(c.numel(18)), stream);
}

int32_t dtype_code(const at::Tensor &t, const char *name)
{
    if (t.scalar_type() == at::kBFloat16) return PSA_OUT_BF16;
    if (t.scalar_type() == at::kFloat) return PSA_OUT_F32;
    throw Refused(std::string(name) + " must be bf16 or f32, not " + name_of(t.scalar_type()));
}

struct Bitmaps {
    const uint32_t *bits = nullptr;
    const int32_t *rows = nullptr;
    int64_t words = 0;
    int32_t count = 0;
    Bitmaps(Call &c, int bits_at, int rows_at, int64_t rows_of_call, int64_t words_of_call, const char *bits_name, const char *rows_name)
    {
        if (c.none(bits_at)) {
            if (!c.none(rows_at)) throw Refused(std::string(rows_name) + " without " + bits_name);
            return;
        }
        const at::Tensor &t = c.tensor(bits_at, bits_name);
        if (t.scalar_type() != at::kInt || t.dim() != 2 || t.size(1) < words_of_call || (t.size(1) > 1 && t.stride(1) != 1))
            throw Refused(std::string(bits_name) + " must be int32 [bitmaps, words >= " + std::to_string(words_of_call) +
                          "], contiguous along the second dimension");
        if (c.none(rows_at) && t.size(0) < rows_of_call) throw Refused(std::string(bits_name) + " needs one bitmap per row, or " + rows_name);
        if (t.size(0) > 0x7fffffff) throw Refused(std::string(bits_name) + " has too many bitmaps");
        bits = static_cast<const uint32_t *>(t.data_ptr());
        words = t.size(0) > 1 ? t.stride(0) : t.size(1);
        count = int32_t(t.size(0));
        rows = c.flat<int32_t>(rows_at, at::kInt, rows_name, rows_of_call);
    }
};

// logits, out, repetition, frequency, presence, history, history_lens, prompt_bits, prompt_rows, bias_indptr, bias_ids, bias_values, mask_bits,
// mask_rows, stream
psa_status_t process_logits(PyObject *const *args, Py_ssize_t given)
{
    Call c(args, given, 15);
    const at::Tensor &logits = c.tensor(0, "logits"), &out = c.tensor(1, "out");
    if (logits.dim() != 2 || out.sizes() != logits.sizes()) throw Refused("logits must be [rows, vocab], and out of the same shape");
    const int32_t in_code = dtype_code(logits, "logits"), out_code = dtype_code(out, "out");
    const int64_t R = logits.size(0), V = logits.size(1), words = (V + 31) / 32;
    if (R > 0x7fffffff || V > 0x7fffffff) throw Refused("logits are too large");
    if (V > 1 && (logits.stride(1) != 1 || out.stride(1) != 1)) throw Refused("logits and out must be contiguous along the vocabulary");
    const int64_t alone = (V + 7) / 8 * 8;   // one row has no stride of its own
    const int64_t in_stride = R > 1 ? logits.stride(0) : alone, out_stride = R > 1 ? out.stride(0) : alone;
    psa_logits_rules_t r{};
    r.repetition = c.flat<float>(2, at::kFloat, "repetition", R);
    r.frequency = c.flat<float>(3, at::kFloat, "frequency", R);
    r.presence = c.flat<float>(4, at::kFloat, "presence", R);
    if (c.none(5) != c.none(6)) throw Refused("history and history_lens go together");
    if (!c.none(5)) {
        const at::Tensor &h = c.tensor(5, "history");
        if (h.scalar_type() != at::kInt || h.dim() != 2 || h.size(0) < R || (h.size(1) > 1 && h.stride(1) != 1) || h.size(1) > 0x7fffffff)
            throw Refused("history must be int32 [rows, capacity], contiguous along the second dimension");
        r.history = static_cast<const int32_t *>(h.data_ptr());
        r.history_stride = h.size(0) > 1 ? h.stride(0) : h.size(1);
        r.history_capacity = int32_t(h.size(1));
        r.history_lens = c.flat<int32_t>(6, at::kInt, "history_lens", R);
    }
    const Bitmaps prompt(c, 7, 8, R, words, "prompt_bits", "prompt_rows"), mask(c, 12, 13, R, words, "mask_bits", "mask_rows");
    r.prompt_bits = prompt.bits; r.prompt_row_words = prompt.words; r.num_prompt_bitmaps = prompt.count; r.prompt_rows = prompt.rows;
    r.mask_bits = mask.bits; r.mask_row_words = mask.words; r.num_mask_bitmaps = mask.count; r.mask_rows = mask.rows;
    if (c.none(9) != c.none(10) || c.none(9) != c.none(11)) throw Refused("bias_indptr, bias_ids and bias_values go together");
    if (!c.none(9)) {
        r.bias_indptr = c.flat<int32_t>(9, at::kInt, "bias_indptr", R + 1);
        r.bias_ids = c.flat<int32_t>(10, at::kInt, "bias_ids");
        const int64_t n = c.numel(10);
        if (n > 0x7fffffff) throw Refused("too many biases");
        r.bias_values = c.flat<float>(11, at::kFloat, "bias_values", n);
        r.num_biases = int32_t(n);
    }
    void *stream = c.stream(14);
    return api.process_logits(logits.data_ptr(), in_code, in_stride, int32_t(R), int32_t(V), &r, out.data_ptr(), out_code, out_stride, stream);
}

// ids, indptr, vocab, bits, stream
psa_status_t mark_tokens(PyObject *const *args, Py_ssize_t given)
{
    Call c(args, given, 5);
    const auto *ids = c.needed<int32_t>(0, at::kInt, "ids");
    const auto *indptr = c.needed<int32_t>(1, at::kInt, "indptr");
    if (c.numel(1) < 1) throw Refused("indptr must hold rows + 1 elements");
    const int64_t n = c.numel(0), rows = c.numel(1) - 1, vocab = c.integer(2), words = (vocab + 31) / 32;
    const at::Tensor &bits = c.tensor(3, "bits");
    if (bits.scalar_type() != at::kInt || bits.dim() != 2 || bits.size(0) < rows || bits.size(1) < words || (bits.size(1) > 1 && bits.stride(1) != 1))
        throw Refused("bits must be int32 [rows, words >= " + std::to_string(words) + "], contiguous along the second dimension");
    if (n > 0x7fffffff || rows > 0x7fffffff || vocab > 0x7fffffff || vocab < 0) throw Refused("sizes must fit 31 bits");
    void *stream = c.stream(4);
    return api.mark_tokens(ids, int32_t(n), indptr, int32_t(rows), int32_t(vocab), static_cast<uint32_t *>(bits.data_ptr()),
                           bits.size(0) > 1 ? bits.stride(0) : bits.size(1), stream);
}

// tensor, type code (0: the tensor's, 1: int32, 2: uint8, 3: float32), sizes, stream, whether it is returned: a new tensor where the given one
// is, allocated for the stream.  A block of the caching allocator belongs to the stream it was allocated on: one of the current stream's may
// still be written by work enqueued there before it was freed, which a call on another stream does not wait for.  What is returned is not given
// back to its stream before the current stream's use of it is over.
PyObject *empty(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        if (n != 5 || !THPVariable_Check(args[0]) || !PyTuple_Check(args[2])) throw Refused("wrong arguments");
        const at::Tensor &like = THPVariable_Unpack(args[0]);
        const long code = PyLong_AsLong(args[1]);
        int64_t sizes[2] = {0, 0};
        const Py_ssize_t dims = PyTuple_GET_SIZE(args[2]);
        if (dims > 2) throw Refused("wrong arguments");
        for (Py_ssize_t i = 0; i < dims; ++i) sizes[i] = PyLong_AsLongLong(PyTuple_GET_ITEM(args[2], i));
        if (PyErr_Occurred()) return nullptr;
        const auto type = code == 1 ? at::kInt : code == 2 ? at::kByte : code == 3 ? at::kFloat : like.scalar_type();
        const auto make = [&] { return at::empty(at::IntArrayRef(sizes, size_t(dims)), at::TensorOptions().dtype(type).device(like.device())); };
        if (!like.is_cuda()) return THPVariable_Wrap(make());
        void *const handle = Call::handle(args[3]);
        const c10::DeviceIndex device = like.get_device();
        const auto current = c10::cuda::getCurrentCUDAStream(device);
        const c10::cuda::CUDAStreamGuard guard(handle ? c10::cuda::getStreamFromExternal(static_cast<cudaStream_t>(handle), device)
                                                      : c10::cuda::getDefaultCUDAStream(device));
        const at::Tensor t = make();
        if (args[4] == Py_True) t.record_stream(current);
        return THPVariable_Wrap(t);
    });
}

// path of the C library, which has been loaded already
PyObject *attach(PyObject *, PyObject *path)
{
    const char *p = PyUnicode_AsUTF8(path);
    if (!p) return nullptr;
    void *lib = dlopen(p, RTLD_NOW | RTLD_LOCAL);
    if (!lib) return PyErr_Format(PyExc_ImportError, "%s", dlerror());
    const struct {
        const char *name;
        void **to;
    } wanted[] = {
        {"psa_build_page_table", reinterpret_cast<void **>(&api.build_page_table)}, {"psa_extend_page_table", reinterpret_cast<void **>(&api.extend_page_table)},
        {"psa_store_kv4", reinterpret_cast<void **>(&api.store_kv4)},               {"psa_load_kv4", reinterpret_cast<void **>(&api.load_kv4)},
        {"psa_decode_kv4", reinterpret_cast<void **>(&api.decode_kv4)},             {"psa_process_logits", reinterpret_cast<void **>(&api.process_logits)},
        {"psa_mark_tokens", reinterpret_cast<void **>(&api.mark_tokens)},
    };
    for (const auto &w : wanted)
        if (!(*w.to = dlsym(lib, w.name))) return PyErr_Format(PyExc_ImportError, "%s lacks %s", p, w.name);
    Py_RETURN_NONE;
}

template <psa_status_t (*body)(PyObject *const *, Py_ssize_t)>
PyMethodDef method(const char *name)
{
    return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&entry<body>)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {
    method<build_page_table>("build_page_table"), method<extend_page_table>("extend_page_table"), method<store_kv4>("store_kv4"),
    method<load_kv4>("load_kv4"), method<decode_kv4>("decode_kv4"), method<process_logits>("process_logits"), method<mark_tokens>("mark_tokens"),
    {"prefix_strides", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&prefix_strides)), METH_FASTCALL, nullptr},
    {"empty", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&empty)), METH_FASTCALL, nullptr},
    {"attach", attach, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_torch_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__torch_calls(void) { return PyModule_Create(&module); }
