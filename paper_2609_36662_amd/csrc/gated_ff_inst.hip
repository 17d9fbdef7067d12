// Launchers of the gated feed-forward block.
#include "gated_ff_kernels.hpp"

namespace autoloco {

namespace {

// launch(first, count) over all workgroups, at most 2^20 at a time.
template <typename Launch>
hipError_t in_slices(int64_t blocks, Launch launch) {
    constexpr int64_t kSlice = int64_t(1) << 20;
    for (int64_t first = 0; first < blocks; first += kSlice) {
        launch((uint32_t)first, dim3((unsigned)(blocks - first < kSlice ? blocks - first : kSlice)));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

Operand along(const MatrixView& m) { return {static_cast<const uint16_t*>(m.data), m.stride, m.rows}; }
Operand across(const MatrixView& m) { return {static_cast<const uint16_t*>(m.data), m.stride, m.cols}; }
MatrixView read(const MatrixOut& m) { return {m.data, m.rows, m.cols, m.stride}; }

template <bool AT, bool BT, bool PAIR, typename Epi>
hipError_t product(const Terms& t, int64_t rows, int64_t cols, const Epi& epi, hipStream_t s) {
    auto grid_of = [&](TileSize size) { return grid_of_product(size, rows, cols, PAIR); };
    bool direct = true;
    int64_t k = 0;
    for (int i = 0; i < t.count; ++i) {
        const Term& x = t.t[i];
        direct = direct && whole_pieces(x.a, x.k, AT) && whole_pieces(x.b, x.k, BT) && reinterpret_cast<uintptr_t>(x.b2) % 16 == 0;
        direct = direct && x.a.stride == t.t[0].a.stride && x.b.stride == t.t[0].b.stride && (i + 1 == t.count || x.k % 64 == 0);
        k += x.k;
    }
    if (!direct) {
        // 64 x 64 where there are fewer tiles of 128 than units (a pair's tile takes at least 128)
        auto through_registers = [&](TileSize size, auto tile) {
            constexpr int T = decltype(tile)::value;
            const Tiles g = grid_of(size);
            return in_slices((int64_t)g.mt * g.nt, [&](uint32_t first, dim3 grid) {
                hipLaunchKernelGGL((product_kernel<Bf16, AT, BT, T, PAIR, Epi>), grid, dim3(256), 0, s, t, rows, cols, g, first, epi);
            });
        };
        const Tiles g = grid_of(TILE_128);
        if constexpr (!PAIR)
            if ((int64_t)g.mt * g.nt < 256) return through_registers(TILE_64, std::integral_constant<int, 1>{});
        return through_registers(TILE_128, std::integral_constant<int, 2>{});
    }
    const TileSize best = tile_of_product(rows, cols, k, PAIR);
    const Tiles g = grid_of(best);
    return with_tile(best, [&](auto tm, auto tn, auto stages) -> hipError_t {
        constexpr int TM = decltype(tm)::value, TN = decltype(tn)::value, ST = decltype(stages)::value;
        if constexpr (PAIR && TN == 1) {
            return hipErrorInvalidValue;   // a pair's tile takes 32 columns of each: not chosen above
        } else {
            return in_slices((int64_t)g.mt * g.nt, [&](uint32_t first, dim3 grid) {
                hipLaunchKernelGGL((direct_kernel<Bf16, AT, BT, TM, TN, ST, PAIR, Epi>), grid, dim3(256), 0, s, t, rows, cols, g, first, epi);
            });
        }
    });
}

Terms one(const Operand& a, const Operand& b, int64_t k, const uint16_t* b2 = nullptr) { return {{{a, b, b2, k}, {}}, 1}; }

template <int ACT>
hipError_t forward(const GatedFf& f, bool tokens, hipStream_t s) {
    const GateEpilogue<ACT> gate{f.h, f.gate, f.up};
    const StoreEpilogue<true> store{f.y};
    const uint16_t* up = static_cast<const uint16_t*>(f.w_up.data);
    const MatrixView h = read(f.h);
    hipError_t e = hipSuccess;
    if (tokens) {
        if (h.cols > 0)
            e = in_slices((h.cols + 15) / 16, [&](uint32_t first, dim3 grid) {
                hipLaunchKernelGGL((tokens_kernel<4, 4, true, GateEpilogue<ACT>>), grid, dim3(4 * 64), 0, s, f.x, along(f.w_gate), up,
                                   first, gate);
            });
        if (e != hipSuccess || f.y.cols == 0) return e;
        // the long sums are fewer: more waves on each
        return in_slices((f.y.cols + 15) / 16, [&](uint32_t first, dim3 grid) {
            hipLaunchKernelGGL((tokens_kernel<16, 4, false, StoreEpilogue<true>>), grid, dim3(16 * 64), 0, s, h, along(f.w_down),
                               static_cast<const uint16_t*>(nullptr), first, store);
        });
    }
    if (h.cols > 0) e = product<false, false, true>(one(along(f.x), along(f.w_gate), f.x.cols, up), h.rows, h.cols, gate, s);
    if (e != hipSuccess || f.y.cols == 0) return e;
    return product<false, false, false>(one(along(h), along(f.w_down), h.cols), f.y.rows, f.y.cols, store, s);
}

template <int ACT>
hipError_t backward(const GatedFfGrad& f, hipStream_t s) {
    const MatrixView dgate = read(f.dgate), dup = read(f.dup);
    auto out = [&](const MatrixOut& to, const Terms& t, auto at, auto bt, bool bf16) -> hipError_t {
        constexpr bool AT = decltype(at)::value, BT = decltype(bt)::value;
        if (to.data == nullptr || to.rows == 0 || to.cols == 0) return hipSuccess;
        return bf16 ? product<AT, BT, false>(t, to.rows, to.cols, StoreEpilogue<true>{to}, s)
                    : product<AT, BT, false>(t, to.rows, to.cols, StoreEpilogue<false>{to}, s);
    };
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    hipError_t e = hipSuccess;
    if (dgate.rows > 0 && dgate.cols > 0)
        e = product<false, true, false>(one(along(f.dy), across(f.w_down), f.dy.cols), dgate.rows, dgate.cols,
                                        GateGradEpilogue<ACT>{f.gate, f.up, f.dgate, f.dup}, s);
    if (e == hipSuccess)
        e = out(f.dx, {{{along(dgate), across(f.w_gate), nullptr, dgate.cols}, {along(dup), across(f.w_up), nullptr, dup.cols}}, 2}, no,
                yes, true);
    if (e == hipSuccess) e = out(f.dw_gate, one(across(dgate), across(f.x), f.x.rows), yes, yes, f.dw_bf16);
    if (e == hipSuccess) e = out(f.dw_up, one(across(dup), across(f.x), f.x.rows), yes, yes, f.dw_bf16);
    if (e == hipSuccess) e = out(f.dw_down, one(across(f.dy), across(f.h), f.x.rows), yes, yes, f.dw_bf16);
    return e;
}

}  // namespace

hipError_t launch_gated_ff(const GatedFf& f, bool tokens, hipStream_t s) {
    return f.activation == kSilu ? forward<kSilu>(f, tokens, s) : forward<kGelu>(f, tokens, s);
}

hipError_t launch_gated_ff_grad(const GatedFfGrad& f, hipStream_t s) {
    return f.activation == kSilu ? backward<kSilu>(f, s) : backward<kGelu>(f, s);
}

}  // namespace autoloco
