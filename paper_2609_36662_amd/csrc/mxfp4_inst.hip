// Launchers of the 4-bit kernels.
#include "mxfp4_tiles.hpp"

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

template <bool BF16>
hipError_t quantize(const MatrixView& x, const Mx4* q, const Mx4* qt, hipStream_t s) {
    if (qt == nullptr) {
        const uint32_t nt = (uint32_t)((q->groups + kRowsGroups - 1) / kRowsGroups);
        return in_slices(nt * ((q->rows + 15) / 16), [&](uint32_t first, dim3 grid) {
            hipLaunchKernelGGL(mx_rows_kernel<BF16>, grid, dim3(kBlock), 0, s, x, *q, nt, first);
        });
    }
    // whole groups of 128 columns, so that the padding is written too
    const uint32_t tiles = (uint32_t)((x.cols + 127) / 128) * (BF16 ? 1 : 2);
    return in_slices(tiles * ((x.rows + 127) / 128), [&](uint32_t first, dim3 grid) {
        if (q != nullptr)
            hipLaunchKernelGGL((mx_cols_kernel<BF16, true>), grid, dim3(kBlock), 0, s, x, *q, *qt, tiles, first);
        else
            hipLaunchKernelGGL((mx_cols_kernel<BF16, false>), grid, dim3(kBlock), 0, s, x, *qt, *qt, tiles, first);
    });
}

template <bool BF16>
hipError_t values(const Mx4& q, const MatrixOut& out, hipStream_t s) {
    const uint32_t nt = (uint32_t)((q.groups + kRowsGroups - 1) / kRowsGroups);
    return in_slices(nt * ((q.rows + kValueRows<BF16> - 1) / kValueRows<BF16>), [&](uint32_t first, dim3 grid) {
        hipLaunchKernelGGL(mx_values_kernel<BF16>, grid, dim3(kBlock), 0, s, q, out, nt, first);
    });
}

// Which tile a product takes: 256 x 256 (one workgroup a compute unit, the most products
// for every byte read from LDS), 128 x 128 (two, or one with four stages on the way where
// there are no more tiles than units and many columns) or 64 x 64.  From the times of full
// and begun rounds of the chip's 256 compute units, in microseconds for g groups of 128
// columns.  Measured (256, 128 and 64): 4,096 x 4,096 x 4,096 39, 40 and 59 us; 4,096 x
// 11,008 x 4,096 110, 115 and 152; 4,608 x 4,096 x 4,096 (a second round barely begun) 61,
// 49 and 65; 2,304 x 4,096 x 4,096 31, 31 and 35; 1,003 x 50,257 x 768 51, 40 and 48; 1,024 x
// 4,096 x 2,048 18.5, 8.7 and 9.7; 512 x 4,096 x 2,048 17.7, 7.8 and 6.4; 2,048 x 2,048 x
// 5,632 37, 19.6 (17.3 with four stages) and 21.5; 768 x 4,096 x 2,048 18.1, 8.3 (8.5) and 8.0.
// Those times are of bf16 results on operands and results that the caches hold.  Where
// they come from memory and large fp32 results go there, the wider tile's longer runs of a
// row count for more (256 and 128): 1,003 x 50,257 x 768 77 and 86 us, 1,024 x 32,768 x
// 768 47 and 55, 2,048 x 32,000 x 2,048 111 and 137 (bf16 results 54 and 61, 31 and 27,
// 94 and 109): a tenth of a microsecond for every megabyte.
enum Tile { TILE_256, TILE_128, TILE_128_DEEP, TILE_64 };
Tile tile_for(int64_t m, int64_t n, int32_t groups, bool bf16) {
    auto tiles = [&](int64_t side) { return ((m + side - 1) / side) * ((n + side - 1) / side); };
    const double g = groups;
    const int64_t t256 = tiles(256), t128 = tiles(128);
    if (t128 < 224) return TILE_64;
    const int64_t full256 = t256 / 256, rest256 = t256 % 256, full128 = t128 / 512, rest128 = t128 % 512;
    const double us256 = full256 * (0.85 * g + 9.0) + (rest256 > 0 ? 0.75 * g + 8.0 : 0.0);
    const double us128 = full128 * (0.52 * g + 3.2) + (rest128 > 256 ? 0.45 * g + 3.0 : rest128 > 0 ? 0.3 * g + 2.0 : 0.0) +
                         (bf16 ? 0.0 : 4e-7 * static_cast<double>(m) * static_cast<double>(n));
    if (us256 < us128) return TILE_256;
    return t128 <= 256 && groups >= 24 ? TILE_128_DEEP : TILE_128;
}

template <int T, int ST, bool BF16>
hipError_t tiles(const Mx4& a, const Mx4& b, const MatrixOut& out, hipStream_t s) {
    const TileGrid g{(uint32_t)((out.rows + 64 * T - 1) / (64 * T)), (uint32_t)((out.cols + 64 * T - 1) / (64 * T))};
    hipLaunchKernelGGL((mx_tile_kernel<T, ST, BF16>), dim3(g.mt * g.nt), dim3(256), 0, s, a, b, out, g);
    return hipGetLastError();
}

template <bool BF16>
hipError_t matmul(const Mx4& a, const Mx4& b, const MatrixOut& out, hipStream_t s) {
    if (a.groups == 0) {
        const int64_t blocks = (out.rows * out.cols + kBlock - 1) / kBlock;
        hipLaunchKernelGGL(zero_matrix_kernel<BF16>, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(kBlock), 0, s, out);
        return hipGetLastError();
    }
    switch (tile_for(out.rows, out.cols, a.groups, BF16)) {
        case TILE_256: return tiles<4, 2, BF16>(a, b, out, s);
        case TILE_128: return tiles<2, 2, BF16>(a, b, out, s);
        case TILE_128_DEEP: return tiles<2, 4, BF16>(a, b, out, s);
        default: return tiles<1, 2, BF16>(a, b, out, s);
    }
}

// Rows of the weight a workgroup takes: 16, 32 or, from 8,193 rows on, 48, the fewest that
// leave no more workgroups than the chip's 256 compute units, so that none waits for a second
// one (13 x 4,096 x 11,008 rows of weight, bf16: 15.8, 15.1 and 9.6 us), with sixteen waves
// where there are few rows to share the columns out over (16 x 11,008 x 4,096 rows: 13.1
// us against 17.0 with eight), eight otherwise.  Each of x's blocks is quantised once a
// workgroup.  From 12,289 rows on there are more workgroups than units (1 and 13 rows of x,
// a call: 2,048 x 32,000 10.9 and 13.6 us, 768 x 50,257 9.7 and 12.9).
// At 17 rows x's form and the tiles take over.  Calls of 16 and 17 rows: 4,096 x 11,008 10.8
// and 13.8 us, 11,008 x 4,096 13.5 and 25.9, 2,048 x 5,632 8.3 and 11.8; where the weight's rows
// are many the tiles would already do at 13 to 16 (2,048 x 32,000 14.1 and 13.2, 768 x
// 50,257 13.1 and 11.7).
template <bool BF16, int R, int NW>
hipError_t tokens_at(const MatrixView& x, const Mx4& w, const MatrixOut& y, hipStream_t s) {
    return in_slices((w.rows + 16 * R - 1) / (16 * R), [&](uint32_t first, dim3 grid) {
        hipLaunchKernelGGL((mx_tokens_kernel<BF16, R, NW>), grid, dim3(NW * 64), 0, s, x, w, y, first);
    });
}
template <bool BF16>
hipError_t tokens(const MatrixView& x, const Mx4& w, const MatrixOut& y, hipStream_t s) {
    if (w.rows <= 16 * 256) return tokens_at<BF16, 1, 16>(x, w, y, s);
    if (w.rows <= 32 * 256) return tokens_at<BF16, 2, 8>(x, w, y, s);
    return tokens_at<BF16, 3, 8>(x, w, y, s);
}

}  // namespace

hipError_t launch_mx_quantize(bool bf16, const MatrixView& x, const Mx4* q, const Mx4* qt, hipStream_t s) {
    return bf16 ? quantize<true>(x, q, qt, s) : quantize<false>(x, q, qt, s);
}

hipError_t launch_mx_values(bool bf16, const Mx4& q, const MatrixOut& out, hipStream_t s) {
    return bf16 ? values<true>(q, out, s) : values<false>(q, out, s);
}

hipError_t launch_mx_matmul(bool bf16, const Mx4& a, const Mx4& b, const MatrixOut& out, hipStream_t s) {
    return bf16 ? matmul<true>(a, b, out, s) : matmul<false>(a, b, out, s);
}

hipError_t launch_mx_tokens(bool bf16, const MatrixView& x, const Mx4& w, const MatrixOut& y, hipStream_t s) {
    return bf16 ? tokens<true>(x, w, y, s) : tokens<false>(x, w, y, s);
}

}  // namespace autoloco
