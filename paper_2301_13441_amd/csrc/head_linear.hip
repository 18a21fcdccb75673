// Dense layers of the trainable head and their gradients, on gfx950 (formulas: head.h).
//
//     linear   z = x weight^T + bias,                            y = residual + scale act(z)
//     gated    (gates | values) = z = x weight^T + bias,         y = act(gates) values
//     gradients, with dz that of z:  grad_x = dz weight,  grad_weight = dz^T x,  grad_bias = sum over rows of dz
//
// Forward is one product whose tiles end in the activation: z goes to memory only where it is wanted.  A gated layer's tile has the same
// columns of gates and of values, in the same lanes.  Backward dz is made in one pass over z and grad, with the sums of its
// columns, and read by two products.  Products of few tiles are cut along the sum's axis; parts are added in a fixed order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "head_flow.hpp"
#include "head_layer.hpp"

namespace head_impl {
namespace {

// ---- forward

// A lane's results of a tile, C = z before the bias, through activation and residual.  WIDE: rows are whole in what a lane stores at a time, and short
// enough that four of them are an offset of 32 bits; ROWS: all rows of the tile are there; KEEP: z is wanted.
template <class T, class S, bool GATED, bool WIDE, bool ROWS, bool KEEP>
__device__ __forceinline__ void finish(const Acc (&c)[S::MT][S::NT], const float (&bias)[S::NT], const End<T> &e, int64_t row0, int64_t column0)
{
    constexpr int N = GATED ? S::NT / 2 : S::NT;  // adjacent columns of y that a lane has
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wave_m = wave / S::WAVES_N, wave_n = wave % S::WAVES_N;
    // Addresses are a wavefront's, which a scalar holds, and a lane's offset from there.
    const int64_t first = row0 + wave_m * (S::MT * 32), column1 = (GATED ? column0 / 2 : column0) + wave_n * (N * 32);
    const int down0 = lane / 32 * 4, across = lane % 32 * N;
    const int rows = static_cast<int>(std::min<int64_t>(S::M, e.n_rows - first)) - down0;
    const int columns = static_cast<int>(std::max<int64_t>(0, std::min<int64_t>(N, e.outs - column1 - across)));
    if (columns == 0) return;
    using Offset = std::conditional_t<WIDE, uint32_t, int64_t>;  // in values
    const int64_t z_columns = GATED ? 2 * e.outs : e.outs;
    const Offset in_y = static_cast<Offset>(down0 * e.outs + across), in_z = static_cast<Offset>(down0 * z_columns + across),
                 in_residual = static_cast<Offset>(down0 * e.residual_stride + across);
    T *y = e.y + first * e.outs + column1;
    T *z = KEEP ? e.z + first * z_columns + column1 : nullptr;
    const T *residual = !GATED && e.residual ? e.residual + first * e.residual_stride + column1 : nullptr;
    // With z, whole rows go past the caches, which z would fill: 16,384 x 1024 bfloat16 to 4096 gated ones 311 us and 281; a training step of these
    // and a linear layer behind them, which reads y, 1424 and 1407, of 4096 rows 477 and 451.  Without z whoever reads y next finds it there: the
    // gated and the linear layer alone 382 us, and 395 past the caches.
    auto put = [&](T *to, const float (&v)[N]) {
        Pack<T, N> p;
#pragma unroll
        for (int k = 0; k < N; ++k) p.v[k] = narrow<T>(v[k]);
        if constexpr (WIDE && sizeof(p) >= 4) {
            using Words = uint32_t __attribute__((ext_vector_type(sizeof(p) / 4)));
            if constexpr (KEEP) __builtin_nontemporal_store(__builtin_bit_cast(Words, p), reinterpret_cast<Words *>(to));
            else *reinterpret_cast<Pack<T, N> *>(to) = p;
        } else if (WIDE) {
            *reinterpret_cast<Pack<T, N> *>(to) = p;
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (k < columns) to[k] = p.v[k];
        }
    };
    with_activation(e.activation, [&](auto ACTIVATION) {
        using Act = Activation<T, ACTIVATION()>;
#pragma unroll
        for (int mt = 0; mt < S::MT; ++mt) {
            // The residual's rows are read 8 at a time: loads do not go past stores, of whose memory nothing is known.
            Pack<T, N> rest[8];
            auto read = [&](int i0) {
#pragma unroll
                for (int i = i0; i < i0 + 8; ++i) {
                    const int down = mt * 32 + i / 4 * 8 + i % 4;
                    if (!ROWS && down >= rows) continue;
                    const T *from = residual + down * e.residual_stride + in_residual;
                    if (WIDE) {
                        rest[i - i0] = *reinterpret_cast<const Pack<T, N> *>(from);
                    } else {
#pragma unroll
                        for (int k = 0; k < N; ++k) rest[i - i0].v[k] = k < columns ? from[k] : T(0);
                    }
                }
            };
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if (!GATED && i % 8 == 0 && residual) read(i);
                const int down = mt * 32 + i / 4 * 8 + i % 4;
                if (!ROWS && down >= rows) continue;
                float v[N];
                if constexpr (GATED) {
                    float gate[N], value[N];
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        gate[k] = c[mt][2 * k][i] + bias[2 * k];
                        value[k] = c[mt][2 * k + 1][i] + bias[2 * k + 1];
                        v[k] = Act(gate[k]).value * value[k];
                    }
                    if constexpr (KEEP) {
                        put(z + down * z_columns + in_z, gate);
                        put(z + (down * z_columns + e.outs) + in_z, value);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < N; ++k) v[k] = c[mt][k][i] + bias[k];
                    if constexpr (KEEP) put(z + down * z_columns + in_z, v);
#pragma unroll
                    for (int k = 0; k < N; ++k) v[k] = e.scale * Act(v[k]).value;
                    if (residual) {
#pragma unroll
                        for (int k = 0; k < N; ++k) v[k] += widen(rest[i % 8].v[k]);
                    }
                }
                put(y + down * e.outs + in_y, v);
            }
        }
    });
}

// Bound by the matrix core where rows and weights are many: 16,384 x 1024 bfloat16 to 4096 gated ones, z kept, 279 us (984 TFLOP/s, with 400 MB of
// results); by the results' way to memory and the activation where the sum is short: 103,069 x 512 bfloat16 to 128, GELU, 39 us (3.4 TB/s); by a
// tile's steps one after the other where tiles are few: 20,011 x 331 float32 to 90, 31 us.
template <class T, class S, bool GATED>
__global__ __launch_bounds__(S::THREADS, 2) void layer_kernel(Operand<T> x, Operand<T> weight, End<T> e, uint32_t row_tiles, uint32_t column_tiles)
{
    extern __shared__ char lds[];
    Flow<T, S, true, true, GATED> flow(x, weight, lds);
    const uint32_t tiles = row_tiles * column_tiles;
    uint32_t ahead = blockIdx.x;
    auto next = [&] {
        if (ahead >= tiles) return;
        uint32_t row_tile, column_tile;
        tile_of(ahead, row_tiles, column_tiles, row_tile, column_tile);
        flow.aim(int64_t{S::M} * row_tile, int64_t{S::N} * column_tile, 0, x.depth);
        ahead += gridDim.x;
    };
    flow.begin(next);
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        uint32_t row_tile, column_tile;
        tile_of(tile, row_tiles, column_tiles, row_tile, column_tile);
        const int64_t column0 = int64_t{S::N} * column_tile, row0 = int64_t{S::M} * row_tile;
        Acc c[S::MT][S::NT];
        flow.run(c, flow.steps_of(0, x.depth), next);
        flow.again(c, row0, column0, 0, x.depth);
        float bias[S::NT] = {};
        if (e.bias) {
#pragma unroll
            for (int nt = 0; nt < S::NT; ++nt) {
                constexpr int N = GATED ? S::NT / 2 : S::NT;
                const int64_t k = (GATED ? column0 / 2 : column0) + S::wave_n() * (N * 32) + threadIdx.x % 32 * N + (GATED ? nt / 2 : nt);
                bias[nt] = k < e.outs ? e.bias[GATED ? k + nt % 2 * e.outs : k] : 0.0f;
            }
        }
        auto end = [&](auto KEEP) {
            if (!e.wide) finish<T, S, GATED, false, false, KEEP()>(c, bias, e, row0, column0);
            else if (row0 + S::M <= e.n_rows) finish<T, S, GATED, true, true, KEEP()>(c, bias, e, row0, column0);
            else finish<T, S, GATED, true, false, KEEP()>(c, bias, e, row0, column0);
        };
        if (e.z) end(std::true_type());
        else end(std::false_type());
    }
}

// Rows of values of 2 bytes that begin at odd ones, into ones that are whole in 16 bytes: a lane makes 16 bytes of 4 or 5 words.  What is behind a
// row's end there is not read by anybody.
__global__ __launch_bounds__(256) void align_kernel(const uint16_t *from, int64_t stride, int64_t n_rows, int dim, uint4 *to, int chunks)
{
    const int64_t n = n_rows * chunks;
    for (int64_t i = int64_t{256} * blockIdx.x + threadIdx.x; i < n; i += int64_t{256} * gridDim.x) {
        const int64_t r = n <= INT32_MAX ? static_cast<int32_t>(i) / chunks : i / chunks;
        const int k = static_cast<int>(i - r * chunks) * 8;
        const uintptr_t first = reinterpret_cast<uintptr_t>(from + r * stride + k), last = reinterpret_cast<uintptr_t>(from + r * stride + dim - 1);
        const bool odd = first & 2;
        const uint32_t *words = reinterpret_cast<const uint32_t *>(first - (odd ? 2 : 0));
        uint32_t w[5];  // those that hold values of the row
#pragma unroll
        for (int j = 0; j < 5; ++j) w[j] = reinterpret_cast<uintptr_t>(words + j) <= last && (j < 4 || odd) ? words[j] : 0;
        uint32_t out[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) out[j] = odd ? __builtin_amdgcn_alignbit(w[j + 1], w[j], 16) : w[j];
        to[i] = make_uint4(out[0], out[1], out[2], out[3]);
    }
}

// The end of a layer whose product came in parts, [splits][n_rows][columns of z] float32: a lane for each value of y.
template <class T, bool GATED>
__global__ __launch_bounds__(256) void finish_kernel(const float *parts, int64_t splits, End<T> e)
{
    const int64_t columns = GATED ? 2 * e.outs : e.outs, n = e.n_rows * e.outs, all = e.n_rows * columns;
    for (int64_t i = int64_t{256} * blockIdx.x + threadIdx.x; i < n; i += int64_t{256} * gridDim.x) {
        const int64_t r = i / e.outs, k = i % e.outs, at = r * columns + k;
        float a = 0, b = 0;
#pragma unroll 4
        for (int64_t s = 0; s < splits; ++s) {
            a += parts[s * all + at];
            if constexpr (GATED) b += parts[s * all + at + e.outs];
        }
        if (e.bias) {
            a += e.bias[k];
            if constexpr (GATED) b += e.bias[e.outs + k];
        }
        if (e.z) {
            e.z[at] = narrow<T>(a);
            if constexpr (GATED) e.z[at + e.outs] = narrow<T>(b);
        }
        with_activation(e.activation, [&](auto ACTIVATION) {
            const float v = Activation<T, ACTIVATION()>(a).value;
            if constexpr (GATED) e.y[i] = narrow<T>(v * b);
            else e.y[i] = narrow<T>(e.scale * v + (e.residual ? widen(e.residual[r * e.residual_stride + k]) : 0.0f));
        });
    }
}

// ---- backward

// dz of `rows` rows from row `rows` * blockIdx.y on, `stride` apart, and parts [gridDim.y][columns] of the sums of its columns, either if
// wanted.  `scale` is only that of the sums.
template <class T>
struct Slopes {
    int32_t activation;
    const T *z, *grad;
    int64_t z_stride, grad_stride;
    int64_t n_rows, outs, rows;
    T *dz;
    int64_t stride;
    float scale;
    float *parts;
};

// dz of bfloat16 values is rounded to bfloat16, one plane of 8 bits: that is what the matrix core takes at once, and a second plane would double the products
// (522 of the 652 us of 16,384 x 1024 to 4096 gated ones), for gradients that are 0.0017 from 64 bits, by their own rounding alone, in place of 0.0023.
// The sums of its columns take it before that.
//
// LANES lanes side by side, of N columns each, 256 / LANES rows at a time.  Bound by memory: 16,384 rows of 4096 gated bfloat16 columns, 671 MB, 118 us
// (5.7 TB/s); one value a lane where rows are odd, 4,099 of 331 gated float32 ones 8.4 us (3.2 TB/s).
template <class T, bool GATED, int N, int LANES>
__global__ __launch_bounds__(256) void slope_kernel(Slopes<T> s)
{
    constexpr int HIGH = 256 / LANES, H = GATED ? 2 : 1;
    __shared__ float lds[HIGH][H][LANES * N];
    const int x = threadIdx.x % LANES, y = threadIdx.x / LANES;
    const int64_t column = (int64_t{LANES} * blockIdx.x + x) * N, columns = H * s.outs;
    const int64_t row0 = s.rows * blockIdx.y, end = std::min(row0 + s.rows, s.n_rows);
    float sums[H][N] = {};
    if (column < s.outs) {
        with_activation(s.activation, [&](auto ACTIVATION) {
            constexpr bool READS = GATED || ACTIVATION() != HEAD_IDENTITY;
            constexpr int ROWS = 4;  // whose loads are on their way together: they do not go past stores, of whose memory nothing is known
            for (int64_t first = row0 + y; first < end; first += ROWS * HIGH) {
                Pack<T, N> g[ROWS], z[ROWS][H];
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const int64_t row = std::min(first + r * HIGH, end - 1);
                    g[r] = *reinterpret_cast<const Pack<T, N> *>(s.grad + row * s.grad_stride + column);
                    if constexpr (READS) {
#pragma unroll
                        for (int h = 0; h < H; ++h) z[r][h] = *reinterpret_cast<const Pack<T, N> *>(s.z + row * s.z_stride + h * s.outs + column);
                    }
                }
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    const int64_t row = first + r * HIGH;
                    if (row >= end) break;
                    Pack<T, N> out[H];
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        float d[H];
                        d[0] = widen(g[r].v[k]);
                        if constexpr (READS) {
                            const Activation<T, ACTIVATION()> a(widen(z[r][0].v[k]));
                            if constexpr (GATED) {
                                d[1] = d[0] * a.value;
                                d[0] *= widen(z[r][1].v[k]);
                            }
                            if constexpr (ACTIVATION() == HEAD_RELU) d[0] = a.slope > 0 ? d[0] : 0;
                            else d[0] *= a.slope;
                        }
#pragma unroll
                        for (int h = 0; h < H; ++h) {
                            sums[h][k] += d[h];
                            out[h].v[k] = narrow<T>(d[h]);
                        }
                    }
                    if (s.dz) {
#pragma unroll
                        for (int h = 0; h < H; ++h) *reinterpret_cast<Pack<T, N> *>(s.dz + row * s.stride + h * s.outs + column) = out[h];
                    }
                }
            }
        });
    }
    if (!s.parts) return;
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
        for (int k = 0; k < N; ++k) lds[y][h][x * N + k] = sums[h][k];
    __syncthreads();
    for (int i = threadIdx.x; i < H * LANES * N; i += 256) {
        const int h = i / (LANES * N), k = i % (LANES * N);
        const int64_t at = int64_t{LANES} * N * blockIdx.x + k;
        float all = 0;
#pragma unroll
        for (int j = 0; j < HIGH; ++j) all += lds[j][h][k];
        if (at < s.outs) s.parts[blockIdx.y * columns + h * s.outs + at] = s.scale * all;
    }
}

// C = A B.  16,384 rows, bfloat16, 8192 columns of dz and 1024 of x: the gradient of x 259 us (1060 TFLOP/s), of the weight 263 in two parts (1045); 4,099
// rows, float32, 662 and 90: 14 us each in 3 and 26 parts, bound by a workgroup's steps.  Each of `splits` parts of the sum's axis goes to a result of its own, [splits][rows][columns] float32; or (out) the one
// part is the result.
template <class T, class S, bool A_ALONG, bool B_ALONG>
__global__ __launch_bounds__(S::THREADS, 2) void sum_kernel(Operand<T> a, Operand<T> b, int64_t columns, uint32_t row_tiles, uint32_t column_tiles,
                                                            uint32_t splits, int64_t split_depth, float scale, float *parts, T *out)
{
    static_assert(!S::NEXT, "a lane's columns are 32 apart");
    extern __shared__ char lds[];
    Flow<T, S, A_ALONG, B_ALONG> flow(a, b, lds);
    const uint32_t tiles = row_tiles * column_tiles * splits;
    uint32_t ahead = blockIdx.x;
    auto place = [&](uint32_t tile, int64_t &row0, int64_t &column0, int64_t &split) {
        uint32_t row_tile, column_tile;
        tile_of(tile, row_tiles * splits, column_tiles, row_tile, column_tile);
        row0 = int64_t{S::M} * (row_tile % row_tiles);
        column0 = int64_t{S::N} * column_tile;
        split = row_tile / row_tiles;
    };
    auto next = [&] {
        if (ahead >= tiles) return;
        int64_t row0, column0, split;
        place(ahead, row0, column0, split);
        flow.aim(row0, column0, split * split_depth, std::min(a.depth, (split + 1) * split_depth));
        ahead += gridDim.x;
    };
    flow.begin(next);
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        int64_t row0, column0, split;
        place(tile, row0, column0, split);
        Acc c[S::MT][S::NT];
        const int64_t from = split * split_depth, to = std::min(a.depth, from + split_depth);
        flow.run(c, flow.steps_of(from, to), next);
        flow.again(c, row0, column0, from, to);
        const int rows = static_cast<int>(std::min<int64_t>(S::M, a.rows - row0)) - S::row(0, 0);
        const int64_t at = (row0 + S::row(0, 0)) * columns + column0 + S::column(0);
        auto each = [&](auto store) {
#pragma unroll
            for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int down = mt * 32 + i / 4 * 8 + i % 4;
#pragma unroll
                    for (int nt = 0; nt < S::NT; ++nt)
                        if (down < rows && column0 + S::column(nt) < columns) store(down * columns + nt * 32, scale * c[mt][nt][i]);
                }
        };
        if (out) {
            T *to = out + at;
            each([&](int64_t k, float v) { to[k] = narrow<T>(v); });
        } else {
            float *to = parts + split * a.rows * columns + at;
            each([&](int64_t k, float v) { to[k] = v; });
        }
    }
}

// ---- what a call launches

// A gated layer's tiles have two columns of z for each of y.
template <class Size>
struct GatedOf;
template <>
struct GatedOf<Tiny> { using Type = Shape<64, 128, 2, 2, false>; };
template <>
struct GatedOf<Small> { using Type = Shape<128, 128, 2, 2, false>; };
template <>
struct GatedOf<Large> { using Type = Shape<256, 256, 4, 2, false>; };

// A linear layer's: a lane has as many adjacent columns of y as its wavefront has 32 of them.
template <class Size>
struct LinearOf { using Type = typename Size::template Of<true>; };
template <>
struct LinearOf<Large> { using Type = Shape<256, 256, 4, 2, true>; };

// Workgroups of a launch: as many as the device holds at a time.  A gated layer's 64 x 128 tiles have 48 KB of LDS, of which a CU holds three.
template <class Size, bool GATED = false>
constexpr int64_t resident_of() { return !std::is_same_v<Size, Tiny> ? Size::RESIDENT : GATED ? 768 : 1024; }

enum { TINY, SMALL, LARGE };

// How a product [rows][columns] over `depth` is cut.
struct Cut {
    int size;
    int64_t row_tiles, column_tiles, splits, split_depth;
    double us;  // by cut_of's model
    int64_t tiles() const { return row_tiles * column_tiles * splits; }
};

// The cut that takes the least time by a model of it, in us, made from times of sum_kernel and of the kernels that add parts over 26 shapes from
// 100 x 64 x 4096 to 8192 x 1024 x 16384: a launch takes 2.2; a workgroup's step `step`, and `more` for each other workgroup that its CU has; a tile's
// end, its results' way to memory, `end`; parts go to memory and back at 4.6 TB/s, in a launch of their own that takes 2.5.  On those shapes
// what this chooses is within 12 % of the fastest cut of all.
//
// A gated layer in one part goes to layer_kernel, whose smallest tile is 64 x 128 and has a price of its own, from that kernel's times over 26 layers, with
// and without z; in parts it goes to sum_kernel like any other product.  On those layers the choice is within 18 % of the fastest, 1.3 % on average:
// bfloat16, z kept, 16,385 x 1024 to 4096 in tiles of 64 x 128, 128 and 256 434, 370 and 300 us, 5000 x 256 to 1024 15.9, 17.1 and 13.8, 2048 x 512 to 256
// 8.9, 10.8 and 17.2; float32 16,384 x 512 to 2048 506 and 439, 4096 x 64 to 128 7.9 and 10.8.
Cut cut_of(int32_t dtype, int64_t rows, int64_t columns, int64_t depth, int most_splits = 256, bool gated = false)
{
    struct Times { double step, more, end; };
    static constexpr Times TIMES[2][3] = {{{0.73, 0.5, 2.0}, {1.54, 1.26, 4.0}, {}}, {{0.39, 0.157, 1.4}, {0.62, 0.33, 3.5}, {1.4, 0, 7.4}}};
    static constexpr Times GATED_TINY[2] = {{1.08, 0.61, 2.75}, {0.56, 0.25, 2.0}};
    constexpr int64_t RESIDENT[] = {resident_of<Tiny>(), resident_of<Small>(), resident_of<Large>()};
    const int64_t step = STEP / value_bytes(dtype);
    const int64_t steps = ceil_div(depth, step);
    const double part_us = static_cast<double>(rows) * columns * 8 / 4.6e6;
    Cut best{};
    double least = INFINITY;
    for (int size = TINY; size <= (dtype == HEAD_BF16 ? LARGE : SMALL); ++size) {
        const int64_t tile = 64 << size, row_tiles = ceil_div(rows, tile);
        for (int splits = 1; splits <= most_splits; splits = splits & (splits - 1) ? splits / 3 * 4 : std::max(splits + 1, splits / 2 * 3)) {  // 1, 2, 3, 4, 6, 8, 12, ..
            const bool wide = gated && size == TINY && splits == 1;
            const auto &t = wide ? GATED_TINY[dtype == HEAD_BF16] : TIMES[dtype == HEAD_BF16][size];
            const int64_t column_tiles = ceil_div(columns, wide ? 128 : tile), tiles = row_tiles * column_tiles * splits;
            const int64_t resident = wide ? resident_of<Tiny, true>() : RESIDENT[size];
            if (splits > 1 && (splits > steps || tiles > 2 * resident || splits * rows * columns > int64_t{1} << 26)) break;
            const int64_t each = splits == 1 ? steps : (static_cast<int32_t>(steps) + splits - 1) / splits;  // of a workgroup
            const double others = static_cast<double>((std::min(tiles, resident) + 255) / 256 - 1);
            const double rounds = static_cast<double>((tiles + resident - 1) / resident);
            const double us = 2.2 + rounds * (static_cast<double>(each) * (t.step + t.more * others) + t.end) + (splits > 1 ? 2.5 + splits * part_us : 0);
            if (us < least) least = us, best = Cut{size, row_tiles, column_tiles, splits, each * step, us};
        }
    }
    best.splits = std::max<int64_t>(1, ceil_div(depth, best.split_depth));  // none is empty
    return best;
}

// The parts of a call's workspace, in bytes from its start.
struct Space {
    int64_t bytes = 0;
    int64_t part(int64_t n)
    {
        const int64_t at = bytes;
        bytes += round_up(n, 256);
        return at;
    }
};

struct Plan : Space {
    int64_t packed;                  // values of a packed row of x and weight
    int64_t x = -1, weight = -1;     // packed operands; -1: used where they are
    Cut forward{}, to_x{}, to_weight{};
    int64_t few = 0;                 // parts of the sum's axis in the kernel for few rows; 0: not by that
    int64_t parts = -1, weight_parts = -1;
    int64_t stride;                  // values of a row of dz
    int64_t dz = -1, bias_rows, bias_chunks, bias_parts = -1;
};

bool whole(int32_t dtype, const void *at, int64_t stride, int64_t n)
{
    const int e = value_bytes(dtype);
    return (address(at) | static_cast<uint64_t>(stride * e) | static_cast<uint64_t>(n * e)) % 16 == 0;
}

// Whether products read an operand where it is: rows begin at words of 4 bytes, not too far apart.
bool readable(int32_t dtype, const void *at, int64_t stride)
{
    const int64_t bytes = stride * value_bytes(dtype);
    return bytes <= FLOW_STRIDE && (address(at) | static_cast<uint64_t>(bytes)) % 4 == 0;
}

constexpr int FORWARD_SPLITS = 32;  // of a layer's product, at most: finish_kernel adds a value's parts one after the other

// Parts of the sum's axis with which the kernel for few rows (head_few.hip) takes a layer whose z has that many columns; 0: tiles take it.
//
// Rows that are whole in 16 bytes, from times of both over 10 shapes from 64 -> 256 to 8192 -> 2048 with 1 to 64 rows: up to 16 rows tiles are faster
// hardly anywhere, but for large bfloat16 weights that the caches hold (1 x 4096 -> 16384 33 us, by tiles 24); with more the few-rows kernel, which
// reads a layer's rows again for each 16 columns, is faster up to some 128 MB of weights times rows (64 x 1024 -> 1024 bfloat16 7.5 us in both, 64 x 2048 ->
// 8192 21.5 and 13.1).  A wavefront's step, of 64 bytes of 16 weights, takes the longer the more rows there are; there are 8 wavefronts in a workgroup, and
// 512 workgroups or more need no other parts.  16 x 16384 -> 64: 30 us in one part, 6.9 in 16.
//
// Others are read value by value, and each of 256 CUs takes its workgroups one after the other: a workgroup by its rows, a step by its loads, fewer than
// 8 steps by their share of 8.  Tiles read such rows in pieces of 16 bytes from any word of 4, bfloat16 rows that begin at odd values after a copy.  From times of
// both over 103 layers, linear and gated, from 3 -> 1000 to 8186 -> 4096 and 31 -> 262144, with 1 to 64 rows: the choice is 1 % behind the faster on
// average, 37 % at most.  us in the few-rows kernel and by tiles, bfloat16: 1 x 58 -> 256 4.0 and 5.7, 1 x 2042 -> 8192 24 and 13, 16 x 4090 -> 16384 156 and 27; odd
// 1 x 249 -> 16384 8.1 and 19, 16 x 4089 -> 16384 154 and 81; float32 16 x 2041 -> 8192 42 and 25.  16 x 1018 -> 1000 bfloat16: 13 in one part, 7.8 in 4.
int64_t few_of(const head_layer &l, int64_t columns, bool gated)
{
    const bool wide = few_wide(l);
    const int64_t row_bytes = l.dim * value_bytes(l.dtype);
    if (l.n_rows > FEW_ROWS || ceil_div(l.n_outputs, FEW_COLUMNS) > FEW_WORKGROUPS) return 0;
    if (l.n_rows > 16 && l.n_rows * columns * row_bytes > int64_t{1} << 27) return 0;
    static const double STEP_US[] = {0.26, 0.42, 0.63, 1.06};
    const double rows = static_cast<double>(l.n_rows);
    const double step = wide ? STEP_US[l.n_rows == 1 ? 0 : l.n_rows <= 16 ? 1 : l.n_rows <= 32 ? 2 : 3] : ((gated ? 2.3 : 1.3) + 0.07 * rows) * 2 / value_bytes(l.dtype);
    const int64_t steps = ceil_div(row_bytes, 64), workgroups = ceil_div(l.n_outputs, FEW_COLUMNS);
    int64_t best = 1;
    double least = INFINITY;
    for (int64_t splits = 1; splits <= 16 && (splits == 1 || (splits * workgroups <= 512 && splits * 8 <= steps)); splits *= 2) {
        double us = static_cast<double>((steps + 8 * splits - 1) / (8 * splits)) * step;
        if (!wide) us = static_cast<double>(ceil_div(splits * workgroups, 256)) * (0.3 + 0.01 * rows + (steps < 8 ? static_cast<double>(steps) / 8 * step : us));
        if (splits > 1) us += 2.4 + 0.1 * static_cast<double>(splits);
        if (splits > 1 && !wide) us = std::max(us, 6.5 + 0.01 * static_cast<double>(splits));  // the host's two launches
        if (us < least) least = us, best = splits;
    }
    if (wide || least < 3.9) return best;  // tiles take more than that by any cut, and looking for the best one takes the host half a microsecond
    double tiles = cut_of(l.dtype, l.n_rows, columns, l.dim, FORWARD_SPLITS, gated).us;
    const int64_t copied = (readable(l.dtype, l.x, l.x_stride) ? 0 : l.n_rows) + (readable(l.dtype, l.weight, l.weight_stride) ? 0 : columns);
    if (copied) tiles += 5 + static_cast<double>(copied * row_bytes) * 2 / 5e6;  // launches, and a copy's reads and writes at 5 TB/s
    return tiles < least ? 0 : best;
}

void plan_operands(const head_layer &l, int64_t columns, Plan &p)
{
    const int e = value_bytes(l.dtype);
    p.packed = round_up(l.dim, 16 / e);
    if (!readable(l.dtype, l.x, l.x_stride)) p.x = p.part(l.n_rows * p.packed * e);
    if (!readable(l.dtype, l.weight, l.weight_stride)) p.weight = p.part(columns * p.packed * e);
}

Plan plan_forward(const head_layer &l, bool gated)
{
    Plan p;
    const int64_t columns = gated ? 2 * l.n_outputs : l.n_outputs;
    if (l.n_rows == 0) return p;
    p.few = few_of(l, columns, gated);
    if (p.few) {
        if (p.few > 1) p.parts = p.part(p.few * l.n_rows * columns * 4);
        return p;
    }
    plan_operands(l, columns, p);
    p.forward = cut_of(l.dtype, l.n_rows, columns, l.dim, FORWARD_SPLITS, gated);
    if (p.forward.splits > 1) p.parts = p.part(p.forward.splits * l.n_rows * columns * 4);
    return p;
}

Plan plan_backward(const head_layer &l, bool gated)
{
    Plan p;
    const int e = value_bytes(l.dtype);
    const int64_t columns = gated ? 2 * l.n_outputs : l.n_outputs;
    if (l.n_rows == 0) return p;
    plan_operands(l, columns, p);
    // Rows a power of two apart would lie in few of the memory's channels: a row more than its values by 256 bytes goes through all.
    p.stride = round_up(columns, 16 / e) + 256 / e;
    p.dz = p.part(l.n_rows * p.stride * e);
    p.bias_chunks = std::min(ceil_div(l.n_rows, 16), ceil_div(1024, ceil_div(l.n_outputs, 64 * 16 / e)));
    p.bias_rows = ceil_div(l.n_rows, p.bias_chunks);
    p.bias_chunks = ceil_div(l.n_rows, p.bias_rows);
    p.bias_parts = p.part(p.bias_chunks * columns * 4);
    p.to_x = cut_of(l.dtype, l.n_rows, l.dim, columns);
    p.to_weight = cut_of(l.dtype, columns, l.dim, l.n_rows);
    if (p.to_x.splits > 1) p.parts = p.part(p.to_x.splits * l.n_rows * l.dim * 4);
    if (p.to_weight.splits > 1) p.weight_parts = p.part(p.to_weight.splits * columns * l.dim * 4);
    return p;
}

template <class S, auto *KERNEL, class... Args>
hipError_t launch_tiles(int64_t tiles, int64_t resident, hipStream_t stream, Args... args)
{
    constexpr size_t BYTES = 2 * (S::M + S::N) * STEP;
    if (const hipError_t e = allow_lds<KERNEL>(BYTES)) return e;
    hipLaunchKernelGGL(KERNEL, grid_of(tiles, resident), dim3(S::THREADS), BYTES, stream, args...);
    return hipGetLastError();
}

// f(the size as a type); float32 products have no large tiles.
template <class T, class F>
hipError_t with_size(int size, F f)
{
    if constexpr (sizeof(T) == 2)
        if (size == LARGE) return f(Large());
    return size == SMALL ? f(Small()) : f(Tiny());
}

// x, or weight, packed if it has to be.
template <class T>
Operand<T> operand(const void *at, int64_t stride, int64_t rows, int64_t dim, int64_t packed, int64_t packed_at, char *workspace, hipStream_t stream)
{
    const T *from = static_cast<const T *>(at);
    if (packed_at < 0) return Operand<T>{from, stride, rows, dim};
    T *to = reinterpret_cast<T *>(workspace + packed_at);
    if constexpr (sizeof(T) == 2)
        hipLaunchKernelGGL(align_kernel, grid_of(ceil_div(rows * packed, 8 * 256)), dim3(256), 0, stream, reinterpret_cast<const uint16_t *>(from), stride, rows,
                           static_cast<int>(dim), reinterpret_cast<uint4 *>(to), static_cast<int>(packed / 8));
    else  // rows too far apart
        hipLaunchKernelGGL((pack_kernel<T>), grid_of(ceil_div(rows * packed, 256)), dim3(256), 0, stream, from, stride, rows, dim, to, packed);
    return Operand<T>{to, packed, rows, dim};
}

template <class T, bool A_ALONG, bool B_ALONG>
hipError_t launch_sum(const Cut &c, const Operand<T> &a, const Operand<T> &b, int64_t columns, float scale, float *parts, T *out, hipStream_t stream)
{
    return with_size<T>(c.size, [&](auto size) {
        using Size = decltype(size);
        using S = typename Size::template Of<false>;
        return launch_tiles<S, sum_kernel<T, S, A_ALONG, B_ALONG>>(c.tiles(), resident_of<Size>(), stream, a, b, columns, static_cast<uint32_t>(c.row_tiles),
                                                                   static_cast<uint32_t>(c.column_tiles), static_cast<uint32_t>(c.splits), c.split_depth,
                                                                   scale, parts, out);
    });
}

template <class T, bool GATED>
hipError_t forward(const head_layer &l, const void *residual, int64_t residual_stride, float scale, void *y, void *z, char *workspace,
                   hipStream_t stream)
{
    const int64_t columns = (GATED ? 2 : 1) * l.n_outputs;
    End<T> end{l.activation, l.bias, static_cast<const T *>(residual), residual ? residual_stride : 0, scale, static_cast<T *>(y), static_cast<T *>(z),
               l.n_rows, l.n_outputs, false};
    const Plan p = plan_forward(l, GATED);
    float *parts = p.parts < 0 ? nullptr : reinterpret_cast<float *>(workspace + p.parts);
    auto finish_parts = [&](int64_t splits) {
        hipLaunchKernelGGL((finish_kernel<T, GATED>), grid_of(ceil_div(l.n_rows * l.n_outputs, 256)), dim3(256), 0, stream, parts, splits, end);
        return hipGetLastError();
    };
    if (p.few) {
        const hipError_t e = launch_few<T, GATED>(l, end, p.few, parts, stream);
        return e || p.few == 1 ? e : finish_parts(p.few);
    }
    const Operand<T> x = operand<T>(l.x, l.x_stride, l.n_rows, l.dim, p.packed, p.x, workspace, stream);
    const Operand<T> weight = operand<T>(l.weight, l.weight_stride, columns, l.dim, p.packed, p.weight, workspace, stream);
    if (const hipError_t e = hipGetLastError()) return e;
    const Cut &c = p.forward;
    if (c.splits > 1) {
        if (const hipError_t e = launch_sum<T, true, true>(c, x, weight, columns, 1.0f, parts, nullptr, stream)) return e;
        return finish_parts(c.splits);
    }
    auto rows_whole = [&](int bytes) {  // in pieces of that many, and four of them in 32 bits of offset
        const uint64_t bits = address(y) | address(z) | address(residual) | static_cast<uint64_t>((l.n_outputs | end.residual_stride) * sizeof(T));
        return bits % bytes == 0 && std::max(2 * l.n_outputs, end.residual_stride) <= int64_t{1} << 26;
    };
    return with_size<T>(c.size, [&](auto size) {
        using Size = decltype(size);
        using S = typename std::conditional_t<GATED, GatedOf<Size>, LinearOf<Size>>::Type;
        end.wide = rows_whole((GATED ? S::NT / 2 : S::NT) * static_cast<int>(sizeof(T)));
        return launch_tiles<S, layer_kernel<T, S, GATED>>(c.tiles(), resident_of<Size, GATED>(), stream, x, weight, end, static_cast<uint32_t>(c.row_tiles),
                                                          static_cast<uint32_t>(c.column_tiles));
    });
}

template <class T, bool GATED>
void launch_slopes(const Slopes<T> &s, int64_t chunks, bool wide, hipStream_t stream)
{
    constexpr int V = 16 / sizeof(T);
    auto run = [&](auto n, auto lanes) {
        hipLaunchKernelGGL((slope_kernel<T, GATED, n(), lanes()>), dim3(static_cast<uint32_t>(ceil_div(s.outs, n() * lanes())), static_cast<uint32_t>(chunks)),
                           dim3(256), 0, stream, s);
    };
    using std::integral_constant;
    const int64_t lanes = wide ? ceil_div(s.outs, V) : s.outs;
    if (wide) {
        if (lanes > 16) run(integral_constant<int, V>(), integral_constant<int, 64>());
        else if (lanes > 4) run(integral_constant<int, V>(), integral_constant<int, 16>());
        else run(integral_constant<int, V>(), integral_constant<int, 4>());
    } else {
        if (lanes > 16) run(integral_constant<int, 1>(), integral_constant<int, 64>());
        else run(integral_constant<int, 1>(), integral_constant<int, 16>());
    }
}

template <class T, bool GATED>
hipError_t backward(const head_layer &l, const void *z, int64_t z_stride, const void *grad, int64_t grad_stride, float scale, void *grad_x,
                    void *grad_weight, float *grad_bias, char *workspace, hipStream_t stream)
{
    const int64_t columns = (GATED ? 2 : 1) * l.n_outputs;
    T *to_x = static_cast<T *>(grad_x), *to_weight = static_cast<T *>(grad_weight);
    if (l.n_rows == 0) {
        hipLaunchKernelGGL((zero_kernel<T>), grid_of(ceil_div(columns * l.dim, 256)), dim3(256), 0, stream, to_weight, columns * l.dim);
        if (grad_bias) hipLaunchKernelGGL((zero_kernel<float>), grid_of(ceil_div(columns, 256)), dim3(256), 0, stream, grad_bias, columns);
        return hipGetLastError();
    }
    const Plan p = plan_backward(l, GATED);
    const Operand<T> x = operand<T>(l.x, l.x_stride, l.n_rows, l.dim, p.packed, p.x, workspace, stream);
    const Operand<T> weight = operand<T>(l.weight, l.weight_stride, columns, l.dim, p.packed, p.weight, workspace, stream);
    // Without an activation dz is grad itself, where products can read it.
    const bool reads = GATED || l.activation != HEAD_IDENTITY;
    const bool makes = reads || !readable(l.dtype, grad, grad_stride);
    const T *dz = static_cast<const T *>(grad);
    int64_t stride = grad_stride;
    if (makes || grad_bias) {
        Slopes<T> s{l.activation, static_cast<const T *>(z), dz, z_stride, grad_stride, l.n_rows, l.n_outputs, p.bias_rows,
                    makes ? reinterpret_cast<T *>(workspace + p.dz) : nullptr, p.stride, scale,
                    grad_bias ? reinterpret_cast<float *>(workspace + p.bias_parts) : nullptr};
        const bool wide = whole(l.dtype, grad, grad_stride, l.n_outputs) && (!reads || whole(l.dtype, z, z_stride, l.n_outputs));
        launch_slopes<T, GATED>(s, p.bias_chunks, wide, stream);
        if (grad_bias) add_parts<float>(s.parts, p.bias_chunks, columns, grad_bias, stream);
        if (makes) dz = s.dz, stride = p.stride;
    }
    if (const hipError_t e = hipGetLastError()) return e;
    float *parts = p.parts < 0 ? nullptr : reinterpret_cast<float *>(workspace + p.parts);
    float *weight_parts = p.weight_parts < 0 ? nullptr : reinterpret_cast<float *>(workspace + p.weight_parts);
    if (const hipError_t e = launch_sum<T, true, false>(p.to_x, Operand<T>{dz, stride, l.n_rows, columns}, Operand<T>{weight.at, weight.stride, weight.depth, columns},
                                                        l.dim, scale, parts, parts ? nullptr : to_x, stream))
        return e;
    if (parts) add_parts(parts, p.to_x.splits, l.n_rows * l.dim, to_x, stream);
    if (const hipError_t e = launch_sum<T, false, false>(p.to_weight, Operand<T>{dz, stride, columns, l.n_rows}, Operand<T>{x.at, x.stride, x.depth, l.n_rows}, l.dim,
                                                         scale, weight_parts, weight_parts ? nullptr : to_weight, stream))
        return e;
    if (weight_parts) add_parts(weight_parts, p.to_weight.splits, columns * l.dim, to_weight, stream);
    return hipGetLastError();
}

}  // namespace

head_layer_launch_t layer_launch(const head_layer &l, bool gated)
{
    const Plan f = plan_forward(l, gated), b = l.n_outputs <= HEAD_MAX_OUTPUTS ? plan_backward(l, gated) : Plan{};
    auto tile = [](const Cut &c) { return c.splits ? 64 << c.size : 0; };
    auto splits = [](const Cut &c) { return static_cast<int32_t>(c.splits); };
    return head_layer_launch_t{static_cast<int32_t>(f.few), f.x >= 0 || b.x >= 0, f.weight >= 0 || b.weight >= 0, tile(f.forward), splits(f.forward),
                               tile(b.to_x), splits(b.to_x), tile(b.to_weight), splits(b.to_weight)};
}

int64_t linear_bytes(const head_layer &l) { return plan_forward(l, false).bytes; }
int64_t gated_bytes(const head_layer &l) { return plan_forward(l, true).bytes; }
int64_t linear_grad_bytes(const head_layer &l) { return plan_backward(l, false).bytes; }
int64_t gated_grad_bytes(const head_layer &l) { return plan_backward(l, true).bytes; }

hipError_t launch_linear(const head_layer &l, const void *residual, int64_t residual_stride, float scale, void *y, void *z, void *workspace,
                         hipStream_t stream)
{
    auto *call = l.dtype == HEAD_F32 ? forward<float, false> : forward<bf16, false>;
    return call(l, residual, residual_stride, scale, y, z, static_cast<char *>(workspace), stream);
}

hipError_t launch_gated(const head_layer &l, void *y, void *z, void *workspace, hipStream_t stream)
{
    auto *call = l.dtype == HEAD_F32 ? forward<float, true> : forward<bf16, true>;
    return call(l, nullptr, 0, 1.0f, y, z, static_cast<char *>(workspace), stream);
}

hipError_t launch_linear_grad(const head_layer &l, const void *z, int64_t z_stride, const void *grad, int64_t grad_stride, float scale,
                              void *grad_x, void *grad_weight, float *grad_bias, void *workspace, hipStream_t stream)
{
    auto *call = l.dtype == HEAD_F32 ? backward<float, false> : backward<bf16, false>;
    return call(l, z, z_stride, grad, grad_stride, scale, grad_x, grad_weight, grad_bias, static_cast<char *>(workspace), stream);
}

hipError_t launch_gated_grad(const head_layer &l, const void *z, int64_t z_stride, const void *grad, int64_t grad_stride, void *grad_x,
                             void *grad_weight, float *grad_bias, void *workspace, hipStream_t stream)
{
    auto *call = l.dtype == HEAD_F32 ? backward<float, true> : backward<bf16, true>;
    return call(l, z, z_stride, grad, grad_stride, 1.0f, grad_x, grad_weight, grad_bias, static_cast<char *>(workspace), stream);
}

}  // namespace head_impl
