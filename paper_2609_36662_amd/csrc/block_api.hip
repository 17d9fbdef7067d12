// Entry points of the feed-forward half of a block: the norms around it, the gated block,
// the orthogonalised step of its matrices.
#include <algorithm>
#include <limits>
#include <memory>

#include "gated_ff_kernels.hpp"
#include "local_checks.hpp"
#include "muon_kernels.hpp"
#include "residual_kernels.hpp"

using namespace autoloco;

namespace {

constexpr int64_t kMaxFf = int64_t(1) << 24;       // rows and widths of a block
constexpr int64_t kMaxMuon = int64_t(1) << 16;     // rows and columns of a matrix
constexpr double kMuonMaxScale = 256.0;            // s at most: the root of rows over columns
// Bytes of X, A and B of a batch, unless one matrix takes more: the more tiles a launch has, the
// less its last round counts (a layer of 4,096 x 11,008 in one batch
// 16.3 ms, in two of at most 1 GiB 17.8).
constexpr int64_t kMuonScratch = int64_t(4) << 30;

// The least eps of a row's mean square that the kernels' fp32 holds to half a rounding step: below, it
// would be rounded coarsely, or to zero, which makes a row of zeros NaN.
constexpr double kLeastEps = 0x1p-126;

// Whether a scalar is finite as the fp32 value that the kernels use.
bool fits(double v) { return std::fabs(v) <= std::numeric_limits<float>::max(); }

// A matrix of rows x cols and dtype (-1: either).
int check_shape(autoloco_ctx* c, const autoloco_matrix& m, const char* name, int64_t rows, int64_t cols, int32_t dtype, bool written) {
    const int st = check_matrix(c, m, name, written);
    if (st != AUTOLOCO_OK) return st;
    if (m.rows != rows || m.cols != cols)
        return fail(c, AUTOLOCO_E_INVALID, std::string(name) + " is " + std::to_string(m.rows) + " x " + std::to_string(m.cols) + ", not " +
                                               std::to_string(rows) + " x " + std::to_string(cols));
    if (dtype >= 0 && m.dtype != dtype) return fail(c, AUTOLOCO_E_INVALID, std::string("wrong dtype of ") + name);
    return AUTOLOCO_OK;
}
// m lies exactly where the input named `as` does: that one is what is written, else m is.
void add_in_place(Buffers& b, const autoloco_matrix& m, const char* name, const autoloco_matrix& in, const char* as) {
    if (m.data == in.data && m.stride == in.stride) {
        for (int i = 0; i < b.n; ++i)
            if (std::strcmp(b.b[i].name, as) == 0) {
                b.b[i].written = true;
                return;
            }
    }
    add_window(b, m, name, true);
}
// Whether an optional matrix is there: of no rows it has no address, but its width.
bool given(const autoloco_matrix& m) { return m.data != nullptr || (m.rows == 0 && m.cols > 0); }
MatrixOut wanted(const autoloco_matrix& m) { return m.data != nullptr ? out_view(m) : MatrixOut{nullptr, 0, 0, 0}; }
MatrixView present(const autoloco_matrix& m) { return m.data != nullptr ? view(m) : MatrixView{nullptr, 0, 0, 0}; }

// What both directions of the block read.
int check_ff(autoloco_ctx* c, const autoloco_feed_forward& f, int64_t out, Buffers& b) {
    constexpr int32_t bf = AUTOLOCO_BF16;
    const int64_t rows = f.x.rows, d = f.x.cols, ffn = f.w_gate.rows;
    int st;
    if (f.activation != AUTOLOCO_SILU && f.activation != AUTOLOCO_GELU) return fail(c, AUTOLOCO_E_INVALID, "unknown activation");
    if ((st = check_shape(c, f.x, "x", rows, d, bf, false)) != AUTOLOCO_OK ||
        (st = check_shape(c, f.w_gate, "w_gate", ffn, d, bf, false)) != AUTOLOCO_OK ||
        (st = check_shape(c, f.w_up, "w_up", ffn, d, bf, false)) != AUTOLOCO_OK ||
        (st = check_shape(c, f.w_down, "w_down", out, ffn, bf, false)) != AUTOLOCO_OK)
        return st;
    if (rows > kMaxFf || d > kMaxFf || ffn > kMaxFf || out > kMaxFf)
        return fail(c, AUTOLOCO_E_INVALID, "rows or a width of more than 2^24");
    if (f.w_gate.stride != f.w_up.stride && ffn > 1) return fail(c, AUTOLOCO_E_INVALID, "w_gate and w_up have different strides");
    add_window(b, f.x, "x", false);
    add_window(b, f.w_gate, "w_gate", false);
    add_window(b, f.w_up, "w_up", false);
    add_window(b, f.w_down, "w_down", false);
    return AUTOLOCO_OK;
}

int check_stream(autoloco_ctx* c, const autoloco_residual& r, const autoloco_matrix& stream, const char* name) {
    int st = check_matrix(c, stream, name, false);
    if (st != AUTOLOCO_OK) return st;
    if (stream.cols > kMaxNormCols) return fail(c, AUTOLOCO_E_INVALID, "more than 2^15 columns");
    if (!fits(r.scale) || !(fits(r.eps) && r.eps >= 0.0))
        return fail(c, AUTOLOCO_E_INVALID, "scale must be finite, eps finite and >= 0 (in fp32)");
    if (r.eps > 0.0 && r.eps < kLeastEps) return fail(c, AUTOLOCO_E_INVALID, "eps between 0 and 2^-126");
    if (given(r.z)) {
        if ((st = check_shape(c, r.z, "z", stream.rows, stream.cols, stream.dtype, false)) != AUTOLOCO_OK) return st;
        if (given(r.gate) && (st = check_shape(c, r.gate, "gate", stream.rows, stream.cols, stream.dtype, false)) != AUTOLOCO_OK)
            return st;
    }
    return AUTOLOCO_OK;
}

}  // namespace

extern "C" {

int autoloco_gated_ff(autoloco_ctx* c, const autoloco_feed_forward* f) {
    return guarded(c, [&]() -> int {
        if (f == nullptr) return fail(c, AUTOLOCO_E_INVALID, "null block");
        constexpr int32_t bf = AUTOLOCO_BF16;
        Buffers b{c};
        int st = check_ff(c, *f, f->y.cols, b);
        if (st != AUTOLOCO_OK) return st;
        const int64_t rows = f->x.rows, ffn = f->w_gate.rows;
        const bool keep = f->gate.data != nullptr;
        if ((st = check_shape(c, f->h, "h", rows, ffn, bf, true)) != AUTOLOCO_OK ||
            (st = check_shape(c, f->y, "y", rows, f->y.cols, bf, true)) != AUTOLOCO_OK)
            return st;
        if (keep != (f->up.data != nullptr)) return fail(c, AUTOLOCO_E_INVALID, "only one of gate and up is kept");
        add_window(b, f->h, "h", true);
        add_window(b, f->y, "y", true);
        if (keep) {
            if ((st = check_shape(c, f->gate, "gate", rows, ffn, bf, true)) != AUTOLOCO_OK ||
                (st = check_shape(c, f->up, "up", rows, ffn, bf, true)) != AUTOLOCO_OK)
                return st;
            add_window(b, f->gate, "gate", true);
            add_window(b, f->up, "up", true);
        }
        if ((st = b.check()) != AUTOLOCO_OK) return st;
        if (rows == 0) return AUTOLOCO_OK;
        const GatedFf a{view(f->x), view(f->w_gate), view(f->w_up), view(f->w_down), out_view(f->y), out_view(f->h),
                        wanted(f->gate), wanted(f->up), f->activation};
        return launched(c, [&] { return launch_gated_ff(a, rows <= AUTOLOCO_FF_TOKENS, c->stream); });
    });
}

int autoloco_gated_ff_grad(autoloco_ctx* c, const autoloco_feed_forward* f, const autoloco_feed_forward_grads* g) {
    return guarded(c, [&]() -> int {
        if (f == nullptr || g == nullptr) return fail(c, AUTOLOCO_E_INVALID, "null block");
        constexpr int32_t bf = AUTOLOCO_BF16;
        Buffers b{c};
        const int64_t out = g->dy.cols;
        int st = check_ff(c, *f, out, b);
        if (st != AUTOLOCO_OK) return st;
        const int64_t rows = f->x.rows, d = f->x.cols, ffn = f->w_gate.rows;
        if ((st = check_shape(c, g->dy, "dy", rows, out, bf, false)) != AUTOLOCO_OK ||
            (st = check_shape(c, f->h, "h", rows, ffn, bf, false)) != AUTOLOCO_OK ||
            (st = check_shape(c, f->gate, "gate", rows, ffn, bf, false)) != AUTOLOCO_OK ||
            (st = check_shape(c, f->up, "up", rows, ffn, bf, false)) != AUTOLOCO_OK ||
            (st = check_shape(c, g->dgate, "dgate", rows, ffn, bf, true)) != AUTOLOCO_OK ||
            (st = check_shape(c, g->dup, "dup", rows, ffn, bf, true)) != AUTOLOCO_OK)
            return st;
        add_window(b, g->dy, "dy", false);
        add_window(b, f->h, "h", false);
        add_window(b, f->gate, "gate", false);
        add_window(b, f->up, "up", false);
        add_in_place(b, g->dgate, "dgate", f->gate, "gate");
        add_in_place(b, g->dup, "dup", f->up, "up");
        if (g->dx.data != nullptr) {
            if ((st = check_shape(c, g->dx, "dx", rows, d, bf, true)) != AUTOLOCO_OK) return st;
            add_window(b, g->dx, "dx", true);
        }
        int32_t dtype = -1;
        const struct {
            const autoloco_matrix& m;
            const char* name;
            int64_t rows, cols;
        } weights[] = {{g->dw_gate, "dw_gate", ffn, d}, {g->dw_up, "dw_up", ffn, d}, {g->dw_down, "dw_down", out, ffn}};
        for (const auto& w : weights) {
            if (w.m.data == nullptr) continue;
            if ((st = check_shape(c, w.m, w.name, w.rows, w.cols, dtype, true)) != AUTOLOCO_OK) return st;
            dtype = w.m.dtype;
            add_window(b, w.m, w.name, true);
        }
        if ((st = b.check()) != AUTOLOCO_OK) return st;
        const GatedFfGrad a{view(f->x),       view(f->w_gate),     view(f->w_up),     view(f->w_down),    view(f->h),
                            view(f->gate),    view(f->up),         view(g->dy),       out_view(g->dgate), out_view(g->dup),
                            wanted(g->dx),    wanted(g->dw_gate),  wanted(g->dw_up),  wanted(g->dw_down), dtype != AUTOLOCO_F32,
                            f->activation};
        return launched(c, [&] { return launch_gated_ff_grad(a, c->stream); });
    });
}

int autoloco_residual_norm(autoloco_ctx* c, const autoloco_residual* r) {
    return guarded(c, [&]() -> int {
        if (r == nullptr) return fail(c, AUTOLOCO_E_INVALID, "null residual");
        int st = check_stream(c, *r, r->x, "x");
        if (st != AUTOLOCO_OK) return st;
        const int64_t rows = r->x.rows, cols = r->x.cols;
        const bool has_z = given(r->z);
        Buffers b{c};
        add_window(b, r->x, "x", false);
        if (has_z) {
            add_window(b, r->z, "z", false);
            if (given(r->gate)) add_window(b, r->gate, "gate", false);
            if (r->z_weight != nullptr) b.add(r->z_weight, cols * 4, "z_weight", 4, false);
            if ((st = check_shape(c, r->out, "out", rows, cols, r->x.dtype, true)) != AUTOLOCO_OK) return st;
            add_in_place(b, r->out, "out", r->x, "x");
        }
        if (r->y.data != nullptr) {
            if ((st = check_shape(c, r->y, "y", rows, cols, r->x.dtype, true)) != AUTOLOCO_OK) return st;
            add_window(b, r->y, "y", true);
            if (r->weight != nullptr) b.add(r->weight, cols * 4, "weight", 4, false);
        }
        if ((st = b.check()) != AUTOLOCO_OK) return st;
        if (rows == 0 || cols == 0 || (!has_z && r->y.data == nullptr)) return AUTOLOCO_OK;
        Residual a{};
        a.x = view(r->x);
        a.z = present(r->z);
        if (has_z) {
            a.gate = present(r->gate);
            a.z_weight = r->z_weight;
            a.out = out_view(r->out);
        }
        a.weight = r->weight;
        a.y = wanted(r->y);
        a.scale = static_cast<float>(r->scale);
        a.eps = static_cast<float>(r->eps);
        return launched(c, [&] { return launch_residual_norm(is_bf16(r->x), a, c->stream); });
    });
}

int64_t autoloco_residual_work(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0 || cols > kMaxNormCols) return 0;
    return 3 * std::min<int64_t>(norm_parts(cols), (std::max<int64_t>(rows, 1) + 3) / 4 * 4) * cols;
}

int autoloco_residual_norm_grad(autoloco_ctx* c, const autoloco_residual* r, const autoloco_residual_grads* g) {
    return guarded(c, [&]() -> int {
        if (r == nullptr || g == nullptr) return fail(c, AUTOLOCO_E_INVALID, "null residual");
        const bool has_z = given(r->z);
        const autoloco_matrix& stream = has_z ? r->out : r->x;
        int st = check_stream(c, *r, stream, has_z ? "out" : "x");
        if (st != AUTOLOCO_OK) return st;
        const int64_t rows = stream.rows, cols = stream.cols;
        const bool gated = has_z && given(r->gate), channel = gated && r->gate.stride == 0;
        if (!has_z && (g->dz.data != nullptr || g->dz_weight != nullptr)) return fail(c, AUTOLOCO_E_INVALID, "dz or dz_weight without z");
        if (!gated && g->dgate.data != nullptr) return fail(c, AUTOLOCO_E_INVALID, "dgate without gate");
        if (g->dz_weight != nullptr && r->z_weight == nullptr) return fail(c, AUTOLOCO_E_INVALID, "dz_weight without z_weight");
        Buffers b{c};
        add_window(b, stream, "out", false);
        if (has_z) add_window(b, r->z, "z", false);
        if (gated) add_window(b, r->gate, "gate", false);
        if (has_z && r->z_weight != nullptr) b.add(r->z_weight, cols * 4, "z_weight", 4, false);
        if (r->weight != nullptr) b.add(r->weight, cols * 4, "weight", 4, false);
        const struct {
            const autoloco_matrix& m;
            const char* name;
        } in[] = {{g->dy, "dy"}, {g->dout, "dout"}};
        for (const auto& i : in) {
            if (i.m.data == nullptr) continue;
            if ((st = check_shape(c, i.m, i.name, rows, cols, stream.dtype, false)) != AUTOLOCO_OK) return st;
            add_window(b, i.m, i.name, false);
        }
        if (g->dx.data != nullptr) {
            if ((st = check_shape(c, g->dx, "dx", rows, cols, stream.dtype, true)) != AUTOLOCO_OK) return st;
            const bool of_dy = g->dy.data == g->dx.data && g->dy.stride == g->dx.stride;
            add_in_place(b, g->dx, "dx", of_dy ? g->dy : g->dout, of_dy ? "dy" : "dout");
        }
        if (g->dz.data != nullptr) {
            if ((st = check_shape(c, g->dz, "dz", rows, cols, stream.dtype, true)) != AUTOLOCO_OK) return st;
            add_window(b, g->dz, "dz", true);
        }
        if (g->dgate.data != nullptr) {
            if ((st = check_shape(c, g->dgate, "dgate", channel ? 1 : rows, cols, stream.dtype, true)) != AUTOLOCO_OK) return st;
            add_window(b, g->dgate, "dgate", true);
        }
        if (g->dweight != nullptr) b.add(g->dweight, cols * 4, "dweight", 4, true);
        if (g->dz_weight != nullptr) b.add(g->dz_weight, cols * 4, "dz_weight", 4, true);
        const bool sums = g->dweight != nullptr || g->dz_weight != nullptr || (channel && g->dgate.data != nullptr);
        if (sums) b.add(g->work, autoloco_residual_work(rows, cols) * 4, "work", 4, true);
        if ((st = b.check()) != AUTOLOCO_OK) return st;
        if (cols == 0 || (rows == 0 && !sums)) return AUTOLOCO_OK;
        ResidualGrad a{};
        a.out = view(stream);
        a.z = present(r->z);
        if (gated) a.gate = view(r->gate);
        a.dy = present(g->dy);
        a.dout = present(g->dout);
        a.weight = r->weight;
        a.z_weight = has_z ? r->z_weight : nullptr;
        a.dx = wanted(g->dx);
        a.dz = wanted(g->dz);
        a.dgate = wanted(g->dgate);
        a.dweight = g->dweight;
        a.dz_weight = g->dz_weight;
        a.work = sums ? g->work : nullptr;
        a.scale = static_cast<float>(r->scale);
        a.eps = static_cast<float>(r->eps);
        a.channel = channel;
        return launched(c, [&] { return launch_residual_grad(is_bf16(stream), a, c->stream); });
    });
}

}  // extern "C"

// ------------------------------------------------------------------ the step --
namespace {

// Device memory that is freed with its owner (which waits for the kernels that use it).
struct DeviceMemory {
    void* p = nullptr;
    ~DeviceMemory() {
        if (p != nullptr) (void)hipFree(p);
    }
};

// Workgroups of a launch over the matrices of one batch.
struct TileRange {
    int64_t first = 0, count = 0;
};
enum TileKind { TILES_NORM, TILES_START, TILES_GRAM, TILES_POLYNOMIAL, TILES_UPDATE, TILE_KINDS };
struct MuonBatch {
    TileRange tiles[TILE_KINDS];
    TileSize size[TILE_KINDS] = {};   // of the products
};
// Rows and columns of tiles of a matrix's product, and its steps of 64 summed elements.
void tiles_of(const MuonMatrix& x, TileKind kind, TileSize size, int64_t& mt, int64_t& nt, int64_t& steps) {
    mt = (x.lda + tile_rows(size) - 1) / tile_rows(size);
    nt = kind == TILES_UPDATE || kind == TILES_START ? (x.ld + tile_cols(size) - 1) / tile_cols(size) : mt;
    steps = (kind == TILES_GRAM ? x.ld : x.lda) / 64;
}
// Appends a matrix's tiles to a launch.  Workgroups go round the eight
// dies (each with a cache of its own): each die gets a run of neighbouring tiles.
void deal(const std::vector<MuonTile>& run, std::vector<MuonTile>& to) {
    const int64_t n = static_cast<int64_t>(run.size());
    const int64_t per = n / 8, extra = n % 8;
    for (int64_t b = 0; b < n; ++b) {
        const int64_t d = b % 8;
        to.push_back(run[d * per + std::min(d, extra) + b / 8]);
    }
}
// The tile of a batch's products: the least time for the tiles of all matrices, each with its
// own steps, as if they were alike.
TileSize tile_for(const std::vector<MuonMatrix>& table, size_t from, size_t to, TileKind kind) {
    TileSize best = TILE_128;
    double least = 1e300;
    for (int k = 0; k < TILE_SIZES; ++k) {
        const TileSize size = static_cast<TileSize>(k);
        if (kind != TILES_UPDATE && tile_rows(size) != tile_cols(size)) continue;   // tiles on one side of the diagonal
        int64_t tiles = 0, longest = 0;
        double sum = 0.0;
        for (size_t i = from; i < to; ++i) {
            int64_t mt, nt, steps;
            tiles_of(table[i], kind, size, mt, nt, steps);
            const int64_t n = kind == TILES_UPDATE ? mt * nt : mt * (mt + 1) / 2;
            tiles += n;
            sum += static_cast<double>(n) * static_cast<double>(steps);
            longest = std::max(longest, steps);
        }
        const double us = std::max(tile_us(size, tiles, sum / static_cast<double>(tiles)), tile_us(size, 1, static_cast<double>(longest)));
        if (us < least) {
            least = us;
            best = size;
        }
    }
    return best;
}

int64_t whole(int64_t n, int64_t unit) { return (n + unit - 1) / unit * unit; }

}  // namespace

struct autoloco_muon {
    int device = 0;
    DeviceMemory matrices, tiles, scratch;
    std::vector<MuonBatch> batches;
};

extern "C" {

int autoloco_muon_create(autoloco_ctx* c, const autoloco_muon_matrix* in, int64_t count, autoloco_muon** out) {
    return guarded(c, [&]() -> int {
        if (out == nullptr || (in == nullptr && count != 0)) return fail(c, AUTOLOCO_E_INVALID, "null list");
        if (count < 0 || count > (1 << 16)) return fail(c, AUTOLOCO_E_INVALID, "count outside 0..2^16");
        std::vector<Buffer> spans;
        std::vector<MuonMatrix> table;
        Buffers one{c};
        for (int64_t i = 0; i < count; ++i) {
            const autoloco_muon_matrix& m = in[i];
            const int64_t rows = m.param.rows, cols = m.param.cols;
            int st;
            if ((st = check_shape(c, m.param, "param", rows, cols, AUTOLOCO_F32, true)) != AUTOLOCO_OK ||
                (st = check_shape(c, m.momentum, "momentum", rows, cols, AUTOLOCO_F32, true)) != AUTOLOCO_OK ||
                (st = check_shape(c, m.grad, "grad", rows, cols, -1, false)) != AUTOLOCO_OK)
                return st;
            if (m.model.data != nullptr && (st = check_shape(c, m.model, "model", rows, cols, AUTOLOCO_BF16, true)) != AUTOLOCO_OK) return st;
            if (rows > kMaxMuon || cols > kMaxMuon) return fail(c, AUTOLOCO_E_INVALID, "a matrix of more than 2^16 rows or columns");
            if (rows == 0 || cols == 0) continue;
            one.n = 0;
            add_window(one, m.param, "a param", true);
            add_window(one, m.momentum, "a momentum", true);
            add_window(one, m.grad, "a grad", false);
            if (m.model.data != nullptr) add_window(one, m.model, "a model", true);
            if ((st = one.check()) != AUTOLOCO_OK) return st;
            spans.insert(spans.end(), one.b, one.b + one.n);
            MuonMatrix x{};
            x.param = static_cast<float*>(m.param.data);
            x.momentum = static_cast<float*>(m.momentum.data);
            x.grad = m.grad.data;
            x.model = static_cast<uint16_t*>(m.model.data);
            x.param_stride = m.param.stride;
            x.momentum_stride = m.momentum.stride;
            x.grad_stride = m.grad.stride;
            x.model_stride = m.model.stride;
            x.rows = static_cast<int32_t>(rows);
            x.cols = static_cast<int32_t>(cols);
            x.tall = rows > cols;
            x.m = static_cast<int32_t>(std::min(rows, cols));
            x.n = static_cast<int32_t>(std::max(rows, cols));
            x.ld = static_cast<int32_t>(whole(x.n, 64));
            x.lda = static_cast<int32_t>(whole(x.m, 64));
            x.grad_bf16 = is_bf16(m.grad);
            x.scale = static_cast<float>(std::exp2(std::round(std::log2(std::sqrt(static_cast<double>(x.n))))));
            x.update = static_cast<float>(0.2 * std::sqrt(static_cast<double>(x.n)));
            x.update_spectral = static_cast<float>(std::sqrt(std::max(1.0, static_cast<double>(rows) / static_cast<double>(cols))));
            x.parts = static_cast<int32_t>(std::min<int64_t>(kMuonParts, (rows * cols + 4095) / 4096));
            table.push_back(x);
        }
        // Among sorted ranges an overlap shows up against the ones that are still open.
        std::sort(spans.begin(), spans.end(), [](const Buffer& a, const Buffer& b) { return a.lo < b.lo; });
        std::vector<const Buffer*> open;
        for (const Buffer& s : spans) {
            open.erase(std::remove_if(open.begin(), open.end(), [&](const Buffer* o) { return o->hi <= s.lo; }), open.end());
            for (const Buffer* o : open)
                if ((o->written || s.written) && overlap(*o, s))
                    return fail(c, AUTOLOCO_E_ALIAS, std::string(s.name) + " overlaps " + o->name);
            open.push_back(&s);
        }
        // Batches, and where each matrix lies in the scratch memory they share.
        auto list = std::make_unique<autoloco_muon>();
        list->device = c->device;
        std::vector<MuonTile> tiles;
        std::vector<size_t> begin;
        int64_t bytes = 0, most = 0;
        std::vector<int64_t> at;
        for (size_t i = 0; i < table.size(); ++i) {
            const MuonMatrix& x = table[i];
            const int64_t of_x = whole(static_cast<int64_t>(x.lda) * x.ld * 2, 256), of_a = whole(static_cast<int64_t>(x.lda) * x.lda * 2, 256);
            const int64_t need = 3 * of_x + 2 * of_a + kMuonParts * 8;
            if (begin.empty() || bytes + need > kMuonScratch) {
                begin.push_back(i);
                bytes = 0;
            }
            at.push_back(bytes);
            bytes += need;
            most = std::max(most, bytes);
        }
        begin.push_back(table.size());
        for (size_t k = 0; k + 1 < begin.size(); ++k) {
            MuonBatch batch;
            std::vector<MuonTile> run;
            // the longest sums first, so that the last tiles to begin are short
            std::vector<size_t> order;
            for (size_t i = begin[k]; i < begin[k + 1]; ++i) order.push_back(i);
            for (int kk = 0; kk < TILE_KINDS; ++kk) {
                const TileKind kind = static_cast<TileKind>(kk);
                const bool product = kind >= TILES_GRAM, square = kind == TILES_GRAM || kind == TILES_POLYNOMIAL;
                if (product) batch.size[kind] = tile_for(table, begin[k], begin[k + 1], kind);
                std::stable_sort(order.begin(), order.end(), [&](size_t a, size_t b) {
                    return kind == TILES_GRAM ? table[a].ld > table[b].ld : table[a].lda > table[b].lda;
                });
                batch.tiles[kind].first = static_cast<int64_t>(tiles.size());
                for (const size_t i : order) {
                    const MuonMatrix& x = table[i];
                    int64_t mt = x.parts, nt = 1, steps;
                    if (kind != TILES_NORM) tiles_of(x, kind, product ? batch.size[kind] : TILE_64, mt, nt, steps);
                    run.clear();
                    for (int64_t band = 0; band < mt; band += 8)
                        for (int64_t tj = 0; tj < (square ? std::min(band + 8, mt) : nt); ++tj)
                            for (int64_t ti = square ? std::max(band, tj) : band; ti < std::min(band + 8, mt); ++ti)
                                run.push_back({static_cast<int32_t>(i), static_cast<uint16_t>(ti), static_cast<uint16_t>(tj)});
                    deal(run, tiles);
                }
                batch.tiles[kind].count = static_cast<int64_t>(tiles.size()) - batch.tiles[kind].first;
            }
            list->batches.push_back(batch);
        }
        if (!table.empty()) {
            DeviceGuard g(c->device);
            if (!g.ok) return fail(c, AUTOLOCO_E_DEVICE, "hipSetDevice failed");
            const size_t table_bytes = table.size() * sizeof(MuonMatrix), tile_bytes = tiles.size() * sizeof(MuonTile);
            if (hipMalloc(&list->scratch.p, most) != hipSuccess || hipMalloc(&list->matrices.p, table_bytes) != hipSuccess ||
                hipMalloc(&list->tiles.p, tile_bytes) != hipSuccess) {
                (void)hipGetLastError();
                return fail(c, AUTOLOCO_E_NOMEM, "the step's scratch memory does not fit device memory");
            }
            for (size_t i = 0; i < table.size(); ++i) {
                MuonMatrix& x = table[i];
                const int64_t of_x = whole(static_cast<int64_t>(x.lda) * x.ld * 2, 256);
                const int64_t of_a = whole(static_cast<int64_t>(x.lda) * x.lda * 2, 256);
                char* p = static_cast<char*>(list->scratch.p) + at[i];
                x.hi[0] = reinterpret_cast<uint16_t*>(p);
                x.hi[1] = reinterpret_cast<uint16_t*>(p + of_x);
                x.lo = reinterpret_cast<uint16_t*>(p + 2 * of_x);
                x.a = reinterpret_cast<uint16_t*>(p + 3 * of_x);
                x.b = reinterpret_cast<uint16_t*>(p + 3 * of_x + of_a);
                x.norm = reinterpret_cast<double*>(p + 3 * of_x + 2 * of_a);
            }
            hipError_t e;
            if ((e = hipMemcpy(list->matrices.p, table.data(), table_bytes, hipMemcpyHostToDevice)) != hipSuccess ||
                (e = hipMemcpy(list->tiles.p, tiles.data(), tile_bytes, hipMemcpyHostToDevice)) != hipSuccess)
                return hip_fail(c, e, "hipMemcpy");
        }
        *out = list.release();
        c->err.clear();
        return AUTOLOCO_OK;
    });
}

void autoloco_muon_destroy(autoloco_muon* l) {
    if (l == nullptr) return;
    DeviceGuard g(l->device);
    delete l;
}

int autoloco_inner_muon(autoloco_ctx* c, autoloco_muon* l, const autoloco_muon_coeffs* k) {
    return guarded(c, [&]() -> int {
        if (l == nullptr || k == nullptr) return fail(c, AUTOLOCO_E_INVALID, "null list or coefficients");
        if (l->device != c->device) return fail(c, AUTOLOCO_E_INVALID, "the list is of another device");
        if (!(std::isfinite(k->lr) && k->lr >= 0.0 && std::isfinite(k->weight_decay) && k->weight_decay >= 0.0 && std::isfinite(k->eps) &&
              k->eps >= 0.0))
            return fail(c, AUTOLOCO_E_INVALID, "lr, weight_decay and eps must be finite and >= 0");
        if (!fits(k->lr * kMuonMaxScale) || !fits(k->lr * k->weight_decay))
            return fail(c, AUTOLOCO_E_INVALID, "lr, or lr times weight_decay, leaves fp32");
        if (!(k->momentum >= 0.0 && k->momentum < 1.0)) return fail(c, AUTOLOCO_E_INVALID, "momentum outside [0, 1)");
        if (k->iterations < 0 || k->iterations > 16) return fail(c, AUTOLOCO_E_INVALID, "iterations outside 0..16");
        if (k->scale != AUTOLOCO_MUON_RMS && k->scale != AUTOLOCO_MUON_SPECTRAL) return fail(c, AUTOLOCO_E_INVALID, "unknown scale");
        return launched(c, [&]() -> hipError_t {
            for (const MuonBatch& b : l->batches) {
                MuonStep s{};
                s.matrices = static_cast<const MuonMatrix*>(l->matrices.p);
                s.momentum = static_cast<float>(k->momentum);
                s.eps = k->eps > 0.0 ? std::max(k->eps, kMuonLeastEps) : 0.0;
                s.lr = static_cast<float>(k->lr);
                s.decay = static_cast<float>(1.0 - k->lr * k->weight_decay);
                s.nesterov = k->nesterov != 0;
                s.spectral = k->scale == AUTOLOCO_MUON_SPECTRAL;
                auto of = [&](TileKind kind) {
                    s.tiles = static_cast<const MuonTile*>(l->tiles.p) + b.tiles[kind].first;
                    return b.tiles[kind].count;
                };
                hipError_t e = launch_muon_momentum(s, of(TILES_NORM), c->stream);
                if (e == hipSuccess) e = launch_muon_start(s, of(TILES_START), c->stream);
                if (e == hipSuccess && k->iterations == 0) e = launch_muon_apply(s, of(TILES_START), c->stream);
                for (int32_t i = 0; i < k->iterations && e == hipSuccess; ++i) {
                    s.from = i & 1;
                    auto product = [&](MuonPhase phase, TileKind kind) {
                        const int64_t blocks = of(kind);
                        return launch_muon_product(phase, b.size[kind], s, blocks, c->stream);
                    };
                    e = product(MUON_GRAM, TILES_GRAM);
                    if (e == hipSuccess) e = product(MUON_POLYNOMIAL, TILES_POLYNOMIAL);
                    if (e == hipSuccess) e = product(i + 1 < k->iterations ? MUON_UPDATE : MUON_FINAL, TILES_UPDATE);
                }
                if (e != hipSuccess) return e;
            }
            return hipSuccess;
        });
    });
}

}  // extern "C"
