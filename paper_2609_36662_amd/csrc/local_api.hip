// Entry points of the operators of a worker's local step: 4-bit linear layers, the
// preference loss, clipping over many tensors.
#include <algorithm>
#include <new>
#include <utility>

#include "clip_kernels.hpp"
#include "context.hpp"
#include "mxfp4_kernels.hpp"
#include "preference_kernels.hpp"

using namespace autoloco;

// A list of gradient tensors, cut into chunks in device memory.
struct autoloco_grads {
    int device = 0;
    int32_t workers = 0;
    int per_cu = 2;   // workgroups a compute unit, over all workers
    GradChunk* chunks = nullptr;
    int64_t first[AUTOLOCO_MAX_K + 1] = {};
    std::vector<Range> ranges;   // the gradients and their packed places, by address; none overlap
};

namespace {

constexpr int64_t kMaxDim = int64_t(1) << 30;
constexpr int64_t kMaxStride = int64_t(1) << 40;
constexpr int64_t kMaxSpan = int64_t(1) << 48;   // elements from a matrix's first to its last

// Columns of a product: a tile's rows lie within 32 bits of its first.
constexpr int64_t kMaxProductCols = int64_t(1) << 24;

// Runs a call's body: memory that runs out on the host is an error like any other.
template <typename Body>
int guarded(autoloco_ctx* c, Body body) {
    if (c == nullptr) return AUTOLOCO_E_INVALID;
    try {
        return body();
    } catch (...) {
        c->err.clear();
        return AUTOLOCO_E_NOMEM;
    }
}

int64_t element_size(int32_t dtype) { return dtype == AUTOLOCO_BF16 ? 2 : 4; }
int64_t groups_of(int64_t cols) { return (cols + 127) / 128; }

// A buffer of a call: what it covers, its alignment, and whether it is written.
struct Buffer {
    uintptr_t lo, hi;
    const char* name;
    uintptr_t align;
    bool written;
};

// The buffers a call is given.  Written ones may overlap nothing else; empty ones
// are not looked at.
struct Buffers {
    autoloco_ctx* ctx;
    Buffer b[12];
    int n = 0;
    void add(const void* p, int64_t bytes, const char* name, uintptr_t align, bool written) {
        if (bytes <= 0) return;
        const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
        b[n++] = {lo, lo + static_cast<uintptr_t>(bytes), name, align, written};
    }
    int check() const {
        for (int i = 0; i < n; ++i) {
            if (b[i].lo == 0) return fail(ctx, AUTOLOCO_E_INVALID, std::string("null ") + b[i].name);
            if (b[i].lo % b[i].align != 0)
                return fail(ctx, AUTOLOCO_E_ALIGN, std::string(b[i].name) + " not aligned to " + std::to_string(b[i].align) + " bytes");
        }
        for (int i = 0; i < n; ++i)
            for (int j = i + 1; j < n; ++j)
                if ((b[i].written || b[j].written) && b[i].lo < b[j].hi && b[j].lo < b[i].hi)
                    return fail(ctx, AUTOLOCO_E_ALIAS, std::string(b[i].name) + " overlaps " + b[j].name);
        for (int i = 0; i < n; ++i) {
            const int st = check_device_ptr(ctx, b[i].lo, b[i].name);
            if (st != AUTOLOCO_OK) return st;
        }
        return AUTOLOCO_OK;
    }
};

int check_matrix(autoloco_ctx* c, const autoloco_matrix& m, const char* name, bool written) {
    if (m.dtype != AUTOLOCO_F32 && m.dtype != AUTOLOCO_BF16)
        return fail(c, AUTOLOCO_E_INVALID, std::string("unknown dtype of ") + name);
    if (m.rows < 0 || m.rows > kMaxDim || m.cols < 0 || m.cols > kMaxDim || m.stride < 0 || m.stride > kMaxStride ||
        (m.rows > 1 && m.stride > (kMaxSpan - m.cols) / (m.rows - 1)))
        return fail(c, AUTOLOCO_E_INVALID, std::string("shape of ") + name + " out of range");
    if (written && m.rows > 1 && m.stride < m.cols)
        return fail(c, AUTOLOCO_E_INVALID, std::string("rows of ") + name + " overlap");
    return AUTOLOCO_OK;
}
int64_t matrix_bytes(const autoloco_matrix& m) {
    if (m.rows == 0 || m.cols == 0) return 0;
    return ((m.rows - 1) * m.stride + m.cols) * element_size(m.dtype);
}
void add_matrix(Buffers& b, const autoloco_matrix& m, const char* name, bool written) {
    b.add(m.data, matrix_bytes(m), name, static_cast<uintptr_t>(element_size(m.dtype)), written);
}
int check_mx(autoloco_ctx* c, const autoloco_mxfp4& q, const char* name) {
    if (q.rows < 0 || q.rows > kMaxDim || q.cols < 0 || q.cols > kMaxDim ||
        q.rows * groups_of(q.cols) >= (int64_t(1) << 31))
        return fail(c, AUTOLOCO_E_INVALID, std::string("shape of ") + name + " out of range");
    return AUTOLOCO_OK;
}
void add_mx(Buffers& b, const autoloco_mxfp4& q, const char* codes, const char* scales, bool written) {
    b.add(q.codes, q.rows * groups_of(q.cols) * 64, codes, 16, written);
    b.add(q.scales, q.rows * groups_of(q.cols) * 4, scales, 4, written);
}

MatrixView view(const autoloco_matrix& m) { return {m.data, m.rows, m.cols, m.stride}; }
MatrixOut out_view(const autoloco_matrix& m) { return {m.data, m.rows, m.cols, m.stride}; }
Mx4 mx_view(const autoloco_mxfp4& q) {
    const int64_t g = groups_of(q.cols);
    return {q.codes, q.scales, q.rows, g * 64, static_cast<int32_t>(g)};
}
bool is_bf16(const autoloco_matrix& m) { return m.dtype == AUTOLOCO_BF16; }

// Launches with the context's device current and its timer running.
template <typename Launch>
int launched(autoloco_ctx* c, Launch launch) {
    DeviceGuard g(c->device);
    if (!g.ok) return fail(c, AUTOLOCO_E_DEVICE, "hipSetDevice failed");
    int st = timer_start(c);
    if (st != AUTOLOCO_OK) return st;
    const hipError_t e = launch();
    if (e != hipSuccess) return hip_fail(c, e, "kernel launch");
    if ((st = timer_stop(c)) != AUTOLOCO_OK) return st;
    c->err.clear();
    return AUTOLOCO_OK;
}

// Checks of a batch of sequences; adds its buffers to b.
int check_sequences(autoloco_ctx* c, const autoloco_sequences* s, Buffers& b) {
    if (s == nullptr) return fail(c, AUTOLOCO_E_INVALID, "null sequences");
    const int st = check_matrix(c, s->logits, "logits", false);
    if (st != AUTOLOCO_OK) return st;
    if (s->sequences < 0 || s->sequences > (1 << 20))
        return fail(c, AUTOLOCO_E_INVALID, "sequences outside 0..2^20");
    const int64_t rows = s->logits.rows;
    add_matrix(b, s->logits, "logits", false);
    b.add(s->labels, rows * 8, "labels", 8, false);
    b.add(s->offsets, (s->sequences + 1) * 8, "offsets", 8, false);
    b.add(s->work, (2 * rows + s->sequences) * 4, "work", 4, true);
    return AUTOLOCO_OK;
}

SequenceArgs sequence_args(const autoloco_sequences* s) {
    SequenceArgs a;
    a.logits = view(s->logits);
    a.labels = s->labels;
    a.offsets = s->offsets;
    a.sequences = s->sequences;
    a.lse = s->work;
    a.logp = s->work + s->logits.rows;
    a.weight = s->work + 2 * s->logits.rows;
    return a;
}

}  // namespace

extern "C" {

int autoloco_mxfp4_quantize(autoloco_ctx* c, const autoloco_matrix* x, const autoloco_mxfp4* q,
                            const autoloco_mxfp4* qt) {
    return guarded(c, [&]() -> int {
        if (x == nullptr || (q == nullptr && qt == nullptr)) return fail(c, AUTOLOCO_E_INVALID, "null matrix");
        int st = check_matrix(c, *x, "x", false);
        if (st != AUTOLOCO_OK) return st;
        Buffers b{c};
        add_matrix(b, *x, "x", false);
        if (q != nullptr) {
            if ((st = check_mx(c, *q, "q")) != AUTOLOCO_OK) return st;
            if (q->rows != x->rows || q->cols != x->cols) return fail(c, AUTOLOCO_E_INVALID, "q has another shape than x");
            add_mx(b, *q, "codes of q", "scales of q", true);
        }
        if (qt != nullptr) {
            if ((st = check_mx(c, *qt, "qt")) != AUTOLOCO_OK) return st;
            if (qt->rows != x->cols || qt->cols != x->rows)
                return fail(c, AUTOLOCO_E_INVALID, "qt has another shape than x transposed");
            add_mx(b, *qt, "codes of qt", "scales of qt", true);
        }
        if ((st = b.check()) != AUTOLOCO_OK) return st;
        if (x->rows == 0 || x->cols == 0) return AUTOLOCO_OK;
        const Mx4 rows = q != nullptr ? mx_view(*q) : Mx4{}, cols = qt != nullptr ? mx_view(*qt) : Mx4{};
        return launched(c, [&] {
            return launch_mx_quantize(is_bf16(*x), view(*x), q != nullptr ? &rows : nullptr,
                                      qt != nullptr ? &cols : nullptr, c->stream);
        });
    });
}

int autoloco_mxfp4_dequantize(autoloco_ctx* c, const autoloco_mxfp4* q, const autoloco_matrix* out) {
    return guarded(c, [&]() -> int {
        if (q == nullptr || out == nullptr) return fail(c, AUTOLOCO_E_INVALID, "null matrix");
        int st = check_mx(c, *q, "q");
        if (st != AUTOLOCO_OK || (st = check_matrix(c, *out, "out", true)) != AUTOLOCO_OK) return st;
        if (q->rows != out->rows || q->cols != out->cols) return fail(c, AUTOLOCO_E_INVALID, "out has another shape than q");
        Buffers b{c};
        add_mx(b, *q, "codes of q", "scales of q", false);
        add_matrix(b, *out, "out", true);
        if ((st = b.check()) != AUTOLOCO_OK) return st;
        if (out->rows == 0 || out->cols == 0) return AUTOLOCO_OK;
        return launched(c, [&] { return launch_mx_values(is_bf16(*out), mx_view(*q), out_view(*out), c->stream); });
    });
}

int autoloco_mxfp4_matmul(autoloco_ctx* c, const autoloco_mxfp4* a, const autoloco_mxfp4* w,
                          const autoloco_matrix* out) {
    return guarded(c, [&]() -> int {
        if (a == nullptr || w == nullptr || out == nullptr) return fail(c, AUTOLOCO_E_INVALID, "null matrix");
        int st = check_mx(c, *a, "a");
        if (st != AUTOLOCO_OK || (st = check_mx(c, *w, "b")) != AUTOLOCO_OK ||
            (st = check_matrix(c, *out, "out", true)) != AUTOLOCO_OK)
            return st;
        if (a->cols != w->cols || out->rows != a->rows || out->cols != w->rows)
            return fail(c, AUTOLOCO_E_INVALID, "shapes do not fit: out[m][n] = sum_k a[m][k] b[n][k]");
        if (a->cols > kMaxProductCols) return fail(c, AUTOLOCO_E_INVALID, "more than 2^24 columns");
        Buffers b{c};
        add_mx(b, *a, "codes of a", "scales of a", false);
        add_mx(b, *w, "codes of b", "scales of b", false);
        add_matrix(b, *out, "out", true);
        if ((st = b.check()) != AUTOLOCO_OK) return st;
        if (out->rows == 0 || out->cols == 0) return AUTOLOCO_OK;
        return launched(c, [&] { return launch_mx_matmul(is_bf16(*out), mx_view(*a), mx_view(*w), out_view(*out), c->stream); });
    });
}

int autoloco_mxfp4_linear(autoloco_ctx* c, const autoloco_matrix* x, const autoloco_mxfp4* w, const autoloco_matrix* y,
                          const autoloco_mxfp4* xq) {
    return guarded(c, [&]() -> int {
        if (x == nullptr || w == nullptr || y == nullptr) return fail(c, AUTOLOCO_E_INVALID, "null matrix");
        int st = check_matrix(c, *x, "x", false);
        if (st != AUTOLOCO_OK || (st = check_mx(c, *w, "w")) != AUTOLOCO_OK ||
            (st = check_matrix(c, *y, "y", true)) != AUTOLOCO_OK)
            return st;
        if (x->cols != w->cols || y->rows != x->rows || y->cols != w->rows)
            return fail(c, AUTOLOCO_E_INVALID, "shapes do not fit: y[m][n] = sum_k x[m][k] w[n][k]");
        if (x->cols > kMaxProductCols) return fail(c, AUTOLOCO_E_INVALID, "more than 2^24 columns");
        if (x->dtype != y->dtype) return fail(c, AUTOLOCO_E_INVALID, "x and y have different dtypes");
        const bool tokens = x->rows <= AUTOLOCO_MXFP4_TOKENS;
        Buffers b{c};
        add_matrix(b, *x, "x", false);
        add_mx(b, *w, "codes of w", "scales of w", false);
        add_matrix(b, *y, "y", true);
        if (!tokens) {
            if (xq == nullptr) return fail(c, AUTOLOCO_E_INVALID, "null xq");
            if ((st = check_mx(c, *xq, "xq")) != AUTOLOCO_OK) return st;
            if (xq->rows != x->rows || xq->cols != x->cols)
                return fail(c, AUTOLOCO_E_INVALID, "xq has another shape than x");
            add_mx(b, *xq, "codes of xq", "scales of xq", true);
        }
        if ((st = b.check()) != AUTOLOCO_OK) return st;
        if (y->rows == 0 || y->cols == 0) return AUTOLOCO_OK;
        return launched(c, [&]() -> hipError_t {
            if (tokens && x->cols > 0) return launch_mx_tokens(is_bf16(*x), view(*x), mx_view(*w), out_view(*y), c->stream);
            Mx4 q = mx_view(*w);   // no columns: nothing is read
            q.rows = x->rows;
            if (x->cols > 0) {
                q = mx_view(*xq);
                const hipError_t e = launch_mx_quantize(is_bf16(*x), view(*x), &q, nullptr, c->stream);
                if (e != hipSuccess) return e;
            }
            return launch_mx_matmul(is_bf16(*y), q, mx_view(*w), out_view(*y), c->stream);
        });
    });
}

int autoloco_sequence_logps(autoloco_ctx* c, const autoloco_sequences* s, float* logps) {
    return guarded(c, [&]() -> int {
        Buffers b{c};
        int st = check_sequences(c, s, b);
        if (st != AUTOLOCO_OK) return st;
        b.add(logps, s->sequences * 4, "logps", 4, true);
        if ((st = b.check()) != AUTOLOCO_OK) return st;
        const SequenceArgs a = sequence_args(s);
        const PreferenceArgs p{nullptr, nullptr, logps, 0.0, 0.0, 0.0};
        return launched(c, [&]() -> hipError_t {
            hipError_t e = hipSuccess;
            if (a.logits.rows > 0) e = launch_row_logp(is_bf16(s->logits), a, c->stream);
            if (e == hipSuccess && a.sequences > 0) e = launch_pairs(a, p, c->stream);
            return e;
        });
    });
}

int autoloco_preference_loss(autoloco_ctx* c, const autoloco_sequences* s, const autoloco_preference* p) {
    return guarded(c, [&]() -> int {
        Buffers b{c};
        int st = check_sequences(c, s, b);
        if (st != AUTOLOCO_OK) return st;
        if (p == nullptr) return fail(c, AUTOLOCO_E_INVALID, "null preference");
        if (s->sequences % 2 != 0) return fail(c, AUTOLOCO_E_INVALID, "an odd number of sequences makes no pairs");
        if (!std::isfinite(p->beta) || !std::isfinite(p->grad_scale) || !(p->smoothing >= 0.0 && p->smoothing <= 1.0))
            return fail(c, AUTOLOCO_E_INVALID, "beta and grad_scale must be finite, smoothing in [0, 1]");
        b.add(p->ref_logps, s->sequences * 4, "ref_logps", 4, false);
        b.add(p->losses, s->sequences / 2 * 4, "losses", 4, true);
        b.add(p->logps, s->sequences * 4, "logps", 4, true);
        const bool grads = p->grads.data != nullptr;
        if (grads) {
            const autoloco_matrix& g = p->grads;
            if ((st = check_matrix(c, g, "grads", true)) != AUTOLOCO_OK) return st;
            if (g.rows != s->logits.rows || g.cols != s->logits.cols || g.dtype != s->logits.dtype)
                return fail(c, AUTOLOCO_E_INVALID, "grads have another shape or dtype than the logits");
            // in place, the logits are what is written
            if (g.data == s->logits.data && g.stride == s->logits.stride) {
                for (int i = 0; i < b.n; ++i)
                    if (std::strcmp(b.b[i].name, "logits") == 0) b.b[i].written = true;
            } else {
                add_matrix(b, g, "grads", true);
            }
        }
        if ((st = b.check()) != AUTOLOCO_OK) return st;
        const SequenceArgs a = sequence_args(s);
        const PreferenceArgs pa{p->ref_logps, p->losses, p->logps, p->beta, p->smoothing, p->grad_scale};
        const bool bf16 = is_bf16(s->logits);
        return launched(c, [&]() -> hipError_t {
            hipError_t e = hipSuccess;
            if (a.logits.rows > 0) e = launch_row_logp(bf16, a, c->stream);
            // The gradient's kernel sees to the pairs itself, each row adding its pair's
            // rows up again, where even a pair that has all the rows costs no more so than
            // a kernel of its own.  How long a pair is only the device knows; one long pair
            // among short ones makes it the square of its rows.  Eight pairs of bf16 rows,
            // all alike and (one with nearly all rows), in the gradient's kernel against
            // apart: 4,096 of 1,000 15.7 us (21.1) against 17.2 (20.2), 8,000 of them 21.7
            // (32.4) against 21.5 (28.0); 2,048 of 4,096 18.0 (18.6) against 18.4 (19.9),
            // 4,096 of them 27.8 (31.6) against 26.0 (29.0); 8,000 of 32,000 252 (270)
            // against 257 (263); of sixteen pairs with 19,456 of 32,000 628 (718) against
            // 630 (652), of 64 with 32,000 of 4,096 164 (401) against 143 (170).
            const bool writes = grads && a.logits.rows > 0 && a.logits.cols > 0;
            const int64_t row_bytes = a.logits.cols * element_size(s->logits.dtype);
            const int64_t most = row_bytes <= 4096 ? 4096 : std::max<int64_t>(2048, row_bytes / 8);
            const bool together = writes && a.sequences > 0 && a.logits.rows <= most;
            if (e == hipSuccess && a.sequences > 0 && !together) e = launch_pairs(a, pa, c->stream);
            if (e == hipSuccess && writes) e = launch_logit_grad(bf16, together, a, pa, out_view(p->grads), c->stream);
            return e;
        });
    });
}

int autoloco_grads_create(autoloco_ctx* c, const autoloco_grad* t, int64_t count, int32_t workers,
                          autoloco_grads** out) {
    return guarded(c, [&]() -> int {
        if (out == nullptr || (t == nullptr && count != 0)) return fail(c, AUTOLOCO_E_INVALID, "null list");
        if (count < 0 || count > (1 << 20)) return fail(c, AUTOLOCO_E_INVALID, "count outside 0..2^20");
        if (workers < 1 || workers > AUTOLOCO_MAX_K) return fail(c, AUTOLOCO_E_INVALID, "workers outside 1..16");
        std::vector<Range> ranges;
        bool packs = false;
        int64_t total = 0;
        for (int64_t i = 0; i < count; ++i) {
            if (t[i].dtype != AUTOLOCO_F32 && t[i].dtype != AUTOLOCO_BF16)
                return fail(c, AUTOLOCO_E_INVALID, "unknown dtype of a gradient");
            if (t[i].n < 0 || t[i].n > (int64_t(1) << 40)) return fail(c, AUTOLOCO_E_INVALID, "n of a gradient outside 0..2^40");
            if (t[i].worker < 0 || t[i].worker >= workers) return fail(c, AUTOLOCO_E_INVALID, "a gradient of no worker");
            if (t[i].n == 0) continue;
            total += t[i].n;
            if (ranges.empty()) packs = t[i].packed != nullptr;
            if ((t[i].packed != nullptr) != packs) return fail(c, AUTOLOCO_E_INVALID, "packed set for some gradients only");
            const uintptr_t g = reinterpret_cast<uintptr_t>(t[i].grad), p = reinterpret_cast<uintptr_t>(t[i].packed);
            if (g == 0) return fail(c, AUTOLOCO_E_INVALID, "null gradient");
            if (g % element_size(t[i].dtype) != 0 || p % 4 != 0)
                return fail(c, AUTOLOCO_E_ALIGN, "a gradient is not aligned to its elements");
            ranges.push_back({g, g + static_cast<uintptr_t>(t[i].n * element_size(t[i].dtype)), "a gradient"});
            if (packs) ranges.push_back({p, p + static_cast<uintptr_t>(t[i].n * 4), "a packed gradient"});
        }
        std::sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
        for (size_t i = 1; i < ranges.size(); ++i)
            if (ranges[i].lo < ranges[i - 1].hi)
                return fail(c, AUTOLOCO_E_ALIAS, std::string(ranges[i].name) + " overlaps " + ranges[i - 1].name);
        DeviceGuard g(c->device);
        if (!g.ok) return fail(c, AUTOLOCO_E_DEVICE, "hipSetDevice failed");
        for (const Range& r : ranges) {
            const int st = check_device_ptr(c, r.lo, r.name);
            if (st != AUTOLOCO_OK) return st;
        }
        autoloco_grads list;
        list.device = c->device;
        list.workers = workers;
        list.ranges = std::move(ranges);
        // Two workgroups a compute unit (two workers' 1.1B bf16 gradients 3.20 ms; 3.72 at one,
        // 3.28 at three or four), three for lists of up to twice the small ones (10M bf16
        // of one worker 19.0 us against 20.9, 18M of four 32.2 against 35.4).
        list.per_cu = total <= 2 * kSmallList ? 3 : 2;
        const int64_t chunk = total <= kSmallList ? kSmallChunk : kChunk;
        std::vector<GradChunk> chunks;
        for (int32_t k = 0; k < workers; ++k) {
            list.first[k] = static_cast<int64_t>(chunks.size());
            for (int64_t i = 0; i < count; ++i) {
                if (t[i].worker != k) continue;
                for (int64_t at = 0; at < t[i].n; at += chunk) {
                    GradChunk ch{};
                    ch.grad = static_cast<char*>(t[i].grad) + at * element_size(t[i].dtype);
                    ch.packed = packs ? t[i].packed + at : nullptr;
                    ch.n = static_cast<int32_t>(std::min<int64_t>(chunk, t[i].n - at));
                    ch.bf16 = t[i].dtype == AUTOLOCO_BF16;
                    chunks.push_back(ch);
                }
            }
        }
        for (int32_t k = workers; k <= AUTOLOCO_MAX_K; ++k) list.first[k] = static_cast<int64_t>(chunks.size());
        auto* l = new autoloco_grads(std::move(list));
        if (!chunks.empty()) {
            const size_t bytes = chunks.size() * sizeof(GradChunk);
            hipError_t e = hipMalloc(&l->chunks, bytes);
            if (e != hipSuccess) {
                delete l;
                (void)hipGetLastError();
                return fail(c, AUTOLOCO_E_NOMEM, "the chunk table does not fit device memory");
            }
            if ((e = hipMemcpy(l->chunks, chunks.data(), bytes, hipMemcpyHostToDevice)) != hipSuccess) {
                (void)hipFree(l->chunks);
                delete l;
                return hip_fail(c, e, "hipMemcpy");
            }
        }
        *out = l;
        c->err.clear();
        return AUTOLOCO_OK;
    });
}

void autoloco_grads_destroy(autoloco_grads* l) {
    if (l == nullptr) return;
    {
        DeviceGuard g(l->device);
        if (l->chunks != nullptr) (void)hipFree(l->chunks);   // waits for the kernels that read it
    }
    delete l;
}

int autoloco_clip_grad_norm(autoloco_ctx* c, autoloco_grads* l, double max_norm, float* norms,
                            autoloco_adamw_stats* out) {
    return guarded(c, [&]() -> int {
        if (l == nullptr) return fail(c, AUTOLOCO_E_INVALID, "null list");
        if (l->device != c->device) return fail(c, AUTOLOCO_E_INVALID, "the list is of another device");
        if (!(std::isfinite(max_norm) && max_norm >= 0.0))
            return fail(c, AUTOLOCO_E_INVALID, "max_norm must be finite and >= 0");
        Buffers b{c};
        if (norms != nullptr) b.add(norms, l->workers * 4, "norms", 4, true);
        int st = b.check();
        if (st != AUTOLOCO_OK) return st;
        if (norms != nullptr) {
            // the first range that ends behind norms' begin
            const auto r = std::upper_bound(l->ranges.begin(), l->ranges.end(), b.b[0].lo,
                                            [](uintptr_t lo, const Range& x) { return lo < x.hi; });
            if (r != l->ranges.end() && r->lo < b.b[0].hi)
                return fail(c, AUTOLOCO_E_ALIAS, std::string("norms overlaps ") + r->name);
        }
        ClipArgs a{};
        a.chunks = l->chunks;
        std::memcpy(a.first, l->first, sizeof(a.first));
        a.partials = c->partials;
        a.max_norm = max_norm;
        a.sums = c->sums;
        a.host_sums = c->host_sums_dev;
        a.norms = norms;
        int64_t most = 1;
        for (int32_t k = 0; k < l->workers; ++k) most = std::max(most, l->first[k + 1] - l->first[k]);
        const int64_t limit = std::max(1, (c->grid_limit > 0 ? std::min(c->grid_limit, 1024) : c->num_cus * l->per_cu) / l->workers);
        const int blocks = static_cast<int>(std::min(most, limit));
        st = launched(c, [&]() -> hipError_t {
            const hipError_t e = launch_tensor_norm(l->workers, blocks, a, c->stream);
            return e != hipSuccess ? e : launch_tensor_clip(l->workers, blocks, a, c->stream);
        });
        if (st != AUTOLOCO_OK || out == nullptr) return st;
        DeviceGuard g(c->device);
        if (!g.ok) return fail(c, AUTOLOCO_E_DEVICE, "hipSetDevice failed");
        if ((st = sums_to_host(c, l->workers)) != AUTOLOCO_OK) return st;
        finish_adamw(c->host_sums, l->workers, max_norm, out);
        return AUTOLOCO_OK;
    });
}

}  // extern "C"
