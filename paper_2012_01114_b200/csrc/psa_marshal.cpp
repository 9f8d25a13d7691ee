// Argument marshalling of the serving entry points, compiled: tensor -> pointer, sizes, strides, the current stream; checks of type, device and layout; outputs that the
// caller does not give.  The same steps in Python take 6 to 8 us a call, longer than the kernels of a single-token step; here about 1.5.  Nothing is computed: every
// function calls the C entry point of its name, whose address bind() is given, and raises PsaError for any status but PSA_OK.
#include <torch/extension.h>

#include <c10/cuda/CUDAStream.h>

#include <string>

#include "../../include/psa.h"

namespace {

decltype(&psa_prompt_attention) g_prompt;
decltype(&psa_cache_append) g_append;
decltype(&psa_cache_attention) g_attention;
decltype(&psa_pages_free) g_free;
decltype(&psa_pages_fork) g_fork;
decltype(&psa_pages_reserve) g_reserve;
decltype(&psa_pages_compact) g_compact;
decltype(&psa_pages_copy) g_copy;
decltype(&psa_cache_append_rotary) g_append_rotary;
decltype(&psa_tree_attention) g_tree;
decltype(&psa_verify_drafts) g_verify;
decltype(&psa_cache_keep) g_keep;
PyObject* g_error;                       // PsaError(status, where)

using at::Tensor;
using Maybe = std::optional<Tensor>;

[[noreturn]] void refuse(const std::string& text) { throw py::value_error(text); }
// Calls an entry point, without the interpreter's lock: the library may be waiting for a stream in another thread (psa_last_issued), and a call then waits for the library.
template <class Entry, class... Args>
void call(const char* where, Entry entry, Args... args) {
    int status;
    {
        py::gil_scoped_release unlocked;
        status = entry(args...);
    }
    if (status == PSA_OK) return;
    PyObject* e = PyObject_CallFunction(g_error, "is", status, where);
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    }
    throw py::error_already_set();
}
int serving_type(const Tensor& t, const char* name) {
    if (t.is_cuda() && t.dim() == 3) {
        if (t.scalar_type() == at::kBFloat16) return PSA_BF16;
        if (t.scalar_type() == at::kHalf) return PSA_F16;
    }
    refuse(std::string(name) + " must be a CUDA tensor [rows, heads, d_k] of bf16 or fp16");
}
int small(int64_t n, const char* name) {
    if (n < 0 || n > 0x7fffffff) refuse(std::string(name) + " is too large");
    return (int)n;
}
// Row stride of a [rows, heads, d] tensor whose heads lie side by side.
long long rows_of(const Tensor& t, const char* name, int64_t heads, int64_t d, const Tensor& like) {
    if (!t.is_cuda() || t.scalar_type() != like.scalar_type() || t.dim() != 3 || t.size(1) != heads || t.size(2) != d ||
        (t.numel() && (t.stride(2) != 1 || (heads > 1 && t.stride(1) != d))))
        refuse(std::string(name) + " must be a CUDA tensor [rows, " + std::to_string(heads) + ", " + std::to_string(d) + "] of Q's or K's type, the heads of a row side by side");
    return t.size(0) > 1 ? t.stride(0) : heads * d;
}
const int* ints(const Tensor& t, const char* name, int64_t count = -1) {
    if (!t.is_cuda() || t.scalar_type() != at::kInt || !t.is_contiguous() || (count >= 0 && t.numel() != count))
        refuse(std::string(name) + " must be a contiguous CUDA tensor of int32" + (count >= 0 ? " with " + std::to_string(count) + " numbers" : std::string()));
    return static_cast<const int*>(t.data_ptr());
}
int* ints_out(const Tensor& t, const char* name, int64_t count = -1) { return const_cast<int*>(ints(t, name, count)); }
void* given(const Tensor& t, const char* name, int64_t rows, int64_t cols, at::ScalarType type) {
    if (!t.is_cuda() || t.scalar_type() != type || !t.is_contiguous() || t.numel() != rows * cols)
        refuse(std::string(name) + " must be a contiguous CUDA tensor [" + std::to_string(rows) + ", " + std::to_string(cols) + "] of type " + c10::toString(type));
    return t.data_ptr();
}
void* stream_of(const std::optional<int64_t>& stream) {
    return stream ? reinterpret_cast<void*>(*stream) : static_cast<void*>(c10::cuda::getCurrentCUDAStream().stream());
}
float scale_of(const std::optional<double>& scale, int64_t d) { return (float)(scale ? *scale : 1.0 / std::sqrt((double)d)); }

Tensor prompt(const Tensor& Q, const Tensor& K, const Tensor& V, const Tensor& q_starts, const Maybe& k_starts, std::optional<double> scale, const Maybe& out, const Maybe& lse,
              std::optional<int64_t> stream) {
    const int type = serving_type(Q, "Q");
    const int64_t rows = Q.size(0), heads = Q.size(1), d = Q.size(2);
    if (K.dim() != 3 || K.size(1) == 0 || heads % K.size(1) || K.sizes() != V.sizes()) refuse("K and V must be [k_rows, kv_heads, d_k] with kv_heads a divisor of Q's heads");
    const int64_t kv_heads = K.size(1), n = q_starts.numel() - 1;
    const long long qs = rows_of(Q, "Q", heads, d, Q), ks = rows_of(K, "K", kv_heads, d, Q), vs = rows_of(V, "V", kv_heads, d, Q);
    Tensor o = out ? *out : at::empty({rows, heads * d}, Q.options());
    call("psa_prompt_attention", g_prompt, Q.data_ptr(), K.data_ptr(), V.data_ptr(), qs, ks, vs, ints(q_starts, "q_starts"), k_starts ? ints(*k_starts, "k_starts", n + 1) : nullptr,
         small(n, "q_starts"), small(rows, "Q"), small(K.size(0), "K"), small(heads, "Q"), (int)kv_heads, small(d, "Q"), scale_of(scale, d), type, given(o, "out", rows, heads * d, Q.scalar_type()),
         lse ? static_cast<float*>(given(*lse, "lse", rows, heads, at::kFloat)) : nullptr, stream_of(stream));
    return o;
}

psa_cache cache_of(const Tensor& pool, const Tensor& tables, const Tensor& lens, int64_t kv_heads, int64_t page_size, int64_t d) {
    if (!pool.is_cuda() || pool.scalar_type() != at::kByte || pool.dim() != 2 || !pool.is_contiguous() || tables.dim() != 2)
        refuse("pool must be a contiguous CUDA tensor [pages, page bytes] of uint8, tables [slots, width]");
    if (pool.size(1) * 16 != kv_heads * page_size * 20 * d)
        refuse("pool pages must have psa_cache_page_bytes(" + std::to_string(kv_heads) + ", " + std::to_string(page_size) + ", " + std::to_string(d) + ") bytes");
    return psa_cache{pool.data_ptr(), ints(tables, "tables"), ints(lens, "lens", tables.size(0)), small(pool.size(0), "pool"), small(tables.size(0), "tables"),
                     small(tables.size(1), "tables"), small(page_size, "page_size"), small(kv_heads, "kv_heads"), small(d, "d_k")};
}

void append(const Tensor& K, const Tensor& V, const Tensor& pool, const Tensor& tables, const Tensor& lens, const Tensor& seqs, const Tensor& starts, int64_t page_size,
            const Maybe& k_held, const Maybe& v_held, std::optional<int64_t> stream) {
    const int type = serving_type(K, "K");
    const int64_t rows = K.size(0), kv_heads = K.size(1), d = K.size(2), n = seqs.numel();
    if (K.sizes() != V.sizes()) refuse("K and V must have one shape");
    const long long ks = rows_of(K, "K", kv_heads, d, K), vs = rows_of(V, "V", kv_heads, d, K);
    const psa_cache cache = cache_of(pool, tables, lens, kv_heads, page_size, d);
    call("psa_cache_append", g_append, &cache, K.data_ptr(), V.data_ptr(), ks, vs, ints(seqs, "seqs"), ints(starts, "starts", n + 1), small(n, "seqs"), small(rows, "K"), type,
         k_held ? given(*k_held, "k_held", rows, kv_heads * d, K.scalar_type()) : nullptr, v_held ? given(*v_held, "v_held", rows, kv_heads * d, K.scalar_type()) : nullptr,
         stream_of(stream));
}

Tensor attention(const Tensor& Q, const Tensor& pool, const Tensor& tables, const Tensor& lens, const Tensor& seqs, const Tensor& q_starts, int64_t kv_heads, int64_t page_size,
                 int64_t max_q, std::optional<double> scale, const Maybe& out, const Maybe& lse, std::optional<int64_t> stream) {
    const int type = serving_type(Q, "Q");
    const int64_t rows = Q.size(0), heads = Q.size(1), d = Q.size(2), n = seqs.numel();
    if (kv_heads <= 0 || heads % kv_heads) refuse("kv_heads must divide Q's heads");
    const long long qs = rows_of(Q, "Q", heads, d, Q);
    const psa_cache cache = cache_of(pool, tables, lens, kv_heads, page_size, d);
    Tensor o = out ? *out : at::empty({rows, heads * d}, Q.options());
    call("psa_cache_attention", g_attention, &cache, Q.data_ptr(), qs, ints(seqs, "seqs"), ints(q_starts, "q_starts", n + 1), small(n, "seqs"), small(rows, "Q"), small(heads, "Q"),
         small(max_q, "max_q"), scale_of(scale, d), type, given(o, "out", rows, heads * d, Q.scalar_type()), lse ? static_cast<float*>(given(*lse, "lse", rows, heads, at::kFloat)) : nullptr,
         stream_of(stream));
    return o;
}

void* dense_like(const Maybe& t, const char* name, int64_t rows, int64_t cols, const Tensor& like) { return t ? given(*t, name, rows, cols, like.scalar_type()) : nullptr; }

std::optional<Tensor> append_rotary(const Tensor& K, const Tensor& V, const Tensor& pool, const Tensor& tables, const Tensor& lens, const Tensor& seqs, const Tensor& starts, int64_t page_size,
                                    const Tensor& freqs, const Maybe& Q, const Maybe& depths, bool interleaved, double amplitude, const Maybe& q_out, const Maybe& k_held, const Maybe& v_held,
                                    std::optional<int64_t> stream) {
    const int type = serving_type(K, "K");
    const int64_t rows = K.size(0), kv_heads = K.size(1), d = K.size(2), n = seqs.numel();
    if (K.sizes() != V.sizes()) refuse("K and V must have one shape");
    if (!freqs.is_cuda() || freqs.scalar_type() != at::kDouble || freqs.dim() != 1 || !freqs.is_contiguous()) refuse("freqs must be a contiguous CUDA tensor [rot / 2] of float64");
    if (Q && (Q->dim() != 3 || Q->size(0) != rows)) refuse("Q must be [rows, heads, d_k] with the rows of K");
    if (!Q && q_out) refuse("q_out is given without Q");
    const long long ks = rows_of(K, "K", kv_heads, d, K), vs = rows_of(V, "V", kv_heads, d, K), qs = Q ? rows_of(*Q, "Q", Q->size(1), d, K) : 0;
    const psa_cache cache = cache_of(pool, tables, lens, kv_heads, page_size, d);
    const psa_rotary rotary = {static_cast<const double*>(freqs.data_ptr()), (float)amplitude, small(2 * freqs.numel(), "freqs"), interleaved};
    std::optional<Tensor> o = q_out;
    if (Q && !o) o = at::empty({rows, Q->size(1), d}, Q->options());
    call("psa_cache_append_rotary", g_append_rotary, &cache, &rotary, Q ? Q->data_ptr() : nullptr, K.data_ptr(), V.data_ptr(), qs, ks, vs, depths ? ints(*depths, "depths", rows) : nullptr,
         ints(seqs, "seqs"), ints(starts, "starts", n + 1), small(n, "seqs"), small(rows, "K"), Q ? small(Q->size(1), "Q") : 0, type,
         Q ? given(*o, "q_out", rows, Q->size(1) * d, K.scalar_type()) : nullptr, dense_like(k_held, "k_held", rows, kv_heads * d, K), dense_like(v_held, "v_held", rows, kv_heads * d, K),
         stream_of(stream));
    return o;
}

Tensor tree(const Tensor& Q, const Tensor& pool, const Tensor& tables, const Tensor& lens, const Tensor& seqs, const Tensor& q_starts, const Tensor& parents, int64_t kv_heads, int64_t page_size,
            int64_t max_q, std::optional<double> scale, const Maybe& out, const Maybe& lse, std::optional<int64_t> stream) {
    const int type = serving_type(Q, "Q");
    const int64_t rows = Q.size(0), heads = Q.size(1), d = Q.size(2), n = seqs.numel();
    if (kv_heads <= 0 || heads % kv_heads) refuse("kv_heads must divide Q's heads");
    const long long qs = rows_of(Q, "Q", heads, d, Q);
    const psa_cache cache = cache_of(pool, tables, lens, kv_heads, page_size, d);
    Tensor o = out ? *out : at::empty({rows, heads * d}, Q.options());
    call("psa_tree_attention", g_tree, &cache, Q.data_ptr(), qs, ints(parents, "parents", rows), ints(seqs, "seqs"), ints(q_starts, "q_starts", n + 1), small(n, "seqs"), small(rows, "Q"),
         small(heads, "Q"), small(max_q, "max_q"), scale_of(scale, d), type, given(o, "out", rows, heads * d, Q.scalar_type()),
         lse ? static_cast<float*>(given(*lse, "lse", rows, heads, at::kFloat)) : nullptr, stream_of(stream));
    return o;
}

// Row stride of [rows, vocab] numbers.
long long vocabulary(const Tensor& t, const char* name, const Tensor& like) {
    if (!t.is_cuda() || t.dim() != 2 || t.sizes() != like.sizes() || t.scalar_type() != like.scalar_type() || (t.numel() && t.size(1) > 1 && t.stride(1) != 1))
        refuse(std::string(name) + " must be a CUDA tensor [rows, vocab] of the logits' shape and type, the numbers of a row side by side");
    return t.size(0) > 1 ? t.stride(0) : t.size(1);
}
std::tuple<Tensor, Tensor, Tensor> verify(const Tensor& logits, const Tensor& tokens, const Tensor& parents, const Tensor& starts, const Tensor& uniform, const Maybe& path, const Maybe& accepted,
                                          const Maybe& next, const Maybe& drafts, const Maybe& temperatures, bool distinct, std::optional<int64_t> stream) {
    if (logits.dim() != 2) refuse("logits must be [rows, vocab]");
    const int64_t rows = logits.size(0), n = starts.numel() - 1;
    const int type = logits.scalar_type() == at::kFloat ? PSA_F32 : logits.scalar_type() == at::kBFloat16 ? PSA_BF16 : logits.scalar_type() == at::kHalf ? PSA_F16 : -1;
    if (type < 0) refuse("logits must be of fp32, bf16 or fp16");
    const long long ls = vocabulary(logits, "logits", logits), ds = drafts ? vocabulary(*drafts, "drafts", logits) : 0;
    const auto numbers = [](const Tensor& t, const char* name, int64_t count) { return static_cast<const float*>(given(t, name, count, 1, at::kFloat)); };
    const auto int_like = starts.options();
    Tensor p = path ? *path : at::empty({rows}, int_like), a = accepted ? *accepted : at::empty({std::max<int64_t>(n, 0)}, int_like), x = next ? *next : at::empty({std::max<int64_t>(n, 0)}, int_like);
    call("psa_verify_drafts", g_verify, logits.data_ptr(), ls, drafts ? drafts->data_ptr() : nullptr, ds, small(logits.size(1), "logits"), type, ints(tokens, "tokens", rows),
         ints(parents, "parents", rows), ints(starts, "starts"), small(n, "starts"), small(rows, "logits"), temperatures ? numbers(*temperatures, "temperatures", n) : nullptr,
         numbers(uniform, "uniform", rows), (int)distinct, ints_out(p, "path", rows), ints_out(a, "accepted", n), ints_out(x, "next", n), stream_of(stream));
    return {p, a, x};
}

void keep(const Tensor& pool, const Tensor& tables, const Tensor& lens, const Tensor& seqs, const Tensor& starts, const Tensor& path, const Tensor& accepted, int64_t kv_heads, int64_t page_size,
          const Maybe& new_lens, std::optional<int64_t> stream) {
    if (!pool.is_cuda() || pool.scalar_type() != at::kByte || !pool.is_contiguous() || (pool.dim() != 2 && pool.dim() != 3) || kv_heads <= 0 || page_size <= 0 ||
        pool.size(-1) % (kv_heads * page_size * 5) || pool.size(-1) / (kv_heads * page_size * 5) * 4 > 0x7fffffff || pool.numel() == 0)
        refuse("pool must be a contiguous CUDA tensor [pages, page bytes] or [layers, pages, page bytes] of uint8, pages of psa_cache_page_bytes(kv_heads, page_size, d_k) bytes");
    const int64_t d = pool.size(-1) / (kv_heads * page_size * 5) * 4, n = seqs.numel();
    const psa_cache cache = cache_of(pool.dim() == 3 ? pool[0] : pool, tables, lens, kv_heads, page_size, d);
    call("psa_cache_keep", g_keep, &cache, pool.dim() == 3 ? small(pool.size(0), "pool") : 1, ints(seqs, "seqs"), ints(starts, "starts", n + 1), ints(path, "path"),
         ints(accepted, "accepted", n), small(n, "seqs"), small(path.numel(), "path"), ints_out(new_lens ? *new_lens : lens, "new_lens", tables.size(0)), stream_of(stream));
}

psa_pages pages_of(const Tensor& tables, const Maybe& lens, const Tensor& refs, int64_t page_size) {
    if (tables.dim() != 2) refuse("tables must be [slots, width]");
    return psa_pages{ints_out(tables, "tables"), lens ? ints_out(*lens, "lens", tables.size(0)) : nullptr, ints_out(refs, "refs"), small(tables.size(0), "tables"),
                     small(tables.size(1), "tables"), small(refs.numel(), "refs"), small(page_size, "page_size")};
}
struct Pool {
    void* at;
    long long page_bytes;
    int layers, pages;
};
// [pages, page bytes] or [layers, pages, page bytes]
Pool pool_of(const Tensor& t, int64_t pages) {
    if (!t.is_cuda() || t.scalar_type() != at::kByte || !t.is_contiguous() || (t.dim() != 2 && t.dim() != 3) || (pages >= 0 && t.size(-2) != pages))
        refuse("a pool must be a contiguous CUDA tensor [pages, page bytes] or [layers, pages, page bytes] of uint8");
    return Pool{t.data_ptr(), t.size(-1), t.dim() == 3 ? small(t.size(0), "pool") : 1, small(t.size(-2), "pool")};
}
void pages_free(const Tensor& tables, const Tensor& lens, const Tensor& refs, const Tensor& seqs, int64_t page_size, std::optional<int64_t> stream) {
    const psa_pages p = pages_of(tables, lens, refs, page_size);
    call("psa_pages_free", g_free, &p, ints(seqs, "seqs"), small(seqs.numel(), "seqs"), stream_of(stream));
}
void pages_fork(const Tensor& tables, const Tensor& lens, const Tensor& refs, const Tensor& parents, const Tensor& children, int64_t page_size, std::optional<int64_t> stream) {
    const psa_pages p = pages_of(tables, lens, refs, page_size);
    call("psa_pages_fork", g_fork, &p, ints(parents, "parents"), ints(children, "children", parents.numel()), small(parents.numel(), "parents"), stream_of(stream));
}
void pages_reserve(const Tensor& tables, const Tensor& lens, const Tensor& refs, const Tensor& pool, const Tensor& seqs, const Tensor& add, int64_t page_size, const Tensor& short_by,
                   std::optional<int64_t> stream) {
    const psa_pages p = pages_of(tables, lens, refs, page_size);
    const Pool q = pool_of(pool, refs.numel());
    call("psa_pages_reserve", g_reserve, &p, q.at, q.page_bytes, q.layers, ints(seqs, "seqs"), ints(add, "add", seqs.numel()), small(seqs.numel(), "seqs"), ints_out(short_by, "short", 1),
         stream_of(stream));
}
void pages_compact(const Tensor& tables, const Tensor& refs, const Tensor& pool, const Tensor& new_tables, const Tensor& new_refs, const Tensor& new_pool, const Tensor& live,
                   std::optional<int64_t> stream) {
    if (new_tables.sizes() != tables.sizes() || new_refs.sizes() != refs.sizes() || new_pool.sizes() != pool.sizes())
        refuse("new_tables, new_refs and new_pool must have the shapes of tables, refs and pool");
    const psa_pages p = pages_of(tables, std::nullopt, refs, 1);
    const Pool q = pool_of(pool, refs.numel()), r = pool_of(new_pool, refs.numel());
    call("psa_pages_compact", g_compact, &p, q.at, q.page_bytes, q.layers, ints_out(new_tables, "new_tables"), ints_out(new_refs, "new_refs"), r.at, ints_out(live, "live", 1), stream_of(stream));
}
void pages_copy(const Tensor& pool, const Tensor& new_pool, const Tensor& src, const Tensor& dst, std::optional<int64_t> stream) {
    const Pool q = pool_of(pool, -1), r = pool_of(new_pool, -1);
    if (q.layers != r.layers || q.page_bytes != r.page_bytes) refuse("both pools must have the same layers and page bytes");
    call("psa_pages_copy", g_copy, q.at, q.pages, r.at, r.pages, q.page_bytes, q.layers, ints(src, "src"), ints(dst, "dst", src.numel()), small(src.numel(), "src"), stream_of(stream));
}

void bind(const std::vector<uintptr_t>& f, py::object error) {
    if (f.size() != 12) refuse("twelve entry points are wanted");
    g_prompt = reinterpret_cast<decltype(g_prompt)>(f[0]);
    g_append = reinterpret_cast<decltype(g_append)>(f[1]);
    g_attention = reinterpret_cast<decltype(g_attention)>(f[2]);
    g_free = reinterpret_cast<decltype(g_free)>(f[3]);
    g_fork = reinterpret_cast<decltype(g_fork)>(f[4]);
    g_reserve = reinterpret_cast<decltype(g_reserve)>(f[5]);
    g_compact = reinterpret_cast<decltype(g_compact)>(f[6]);
    g_copy = reinterpret_cast<decltype(g_copy)>(f[7]);
    g_append_rotary = reinterpret_cast<decltype(g_append_rotary)>(f[8]);
    g_tree = reinterpret_cast<decltype(g_tree)>(f[9]);
    g_verify = reinterpret_cast<decltype(g_verify)>(f[10]);
    g_keep = reinterpret_cast<decltype(g_keep)>(f[11]);
    g_error = error.release().ptr();
}

}  // namespace

PYBIND11_MODULE(psa_marshal, m) {
    m.def("bind", &bind);
    m.def("prompt", &prompt);
    m.def("append", &append);
    m.def("attention", &attention);
    m.def("append_rotary", &append_rotary);
    m.def("tree", &tree);
    m.def("verify", &verify);
    m.def("keep", &keep);
    m.def("pages_free", &pages_free);
    m.def("pages_fork", &pages_fork);
    m.def("pages_reserve", &pages_reserve);
    m.def("pages_compact", &pages_compact);
    m.def("pages_copy", &pages_copy);
}
