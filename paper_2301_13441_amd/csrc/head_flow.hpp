// The products of head_linear.hip, on gfx950: the shapes and the layout in LDS of head_product.hpp, with the matrix core fed across the steps of
// the sum and across tiles.
//
// A step's tiles of A and B are loaded two steps ahead, into the half of LDS that a step has just left.  A wavefront reads the next 32
// bytes of the sum's axis while the matrix core works on the last ones, over the end of a step too: the barrier, the loads that it
// lets go and the next step's first reads come before a step's last instructions of the matrix core, so that it has work meanwhile.
//
// Products of float32 values go to the matrix core as products of bfloat16 ones, for which its rate is sixteen times that for float32: a value is
// the sum of three of 8 bits each, exactly, and of the nine products of two values' parts the three smallest, together below 2^-25 of the
// whole, are left out, which is half of what a float32 product is rounded by.  The parts are made of what a wavefront has read, 11 vector
// instructions for two values.  bfloat16 has nothing below 2^-133, so values below 2^-109 lose bits.  Infinite values, and the few that round to
// one, have no such parts: a sum that is not finite in the end is made again, with float32 instructions (again).
//
// Loads go through buffer descriptors, of 16 bytes that begin at any word of 4, whose bounds give zeros past the last row and past the end of a sum that lies across memory, and by which a
// lane has one 32-bit offset for all its loads of an operand.
#pragma once

#include "head_product.hpp"

namespace head_impl {
namespace {

constexpr int64_t FLOW_STRIDE = (1 << 21) + 256;  // bytes of a row's step, at most: offsets in a tile, of up to 256 rows, stay far below 2^31

// Tiles of ROWS x 128 bytes of an operand: layout in LDS and meaning of the parameters as in Tile.  PAIRS: the operand's rows are two halves, of
// which a lane is to have the same ones: row nt * 32 + l of every NT * 32 is row NT / 2 * l + nt / 2 of the tile's ROWS / 2 of half nt % 2.
template <class T, bool ALONG, int ROWS, int THREADS, int NT, bool PAIRS, int FRAGMENTS>
struct FlowTile {
    static constexpr int VALUES = 16 / sizeof(T), DEPTH = STEP / sizeof(T), BYTES = ROWS * STEP, LOADS = BYTES / (THREADS * 16), WAVES = THREADS / 64;
    static constexpr int SLOTS = ALONG ? STEP / 16 : ROWS / VALUES;  // chunks of a row of the tile
    static constexpr int EACH = 64 / SLOTS;                          // rows that a wavefront loads at a time
    static constexpr int ADDRESSES = ALONG ? STEP / 32 : FRAGMENTS;
    static_assert(LOADS > 0, "every lane has a chunk of a step");

    static __device__ __forceinline__ int key(int r)
    {
        if constexpr (ALONG) return r / (256 / STEP) % SLOTS;
        if constexpr (sizeof(T) == 4) return r / 4 % 2 * 8;
        return ROWS >= 128 ? r % 4 * 4 : r / 2 % 2 * 4;
    }

    uint32_t lane_offset;  // bytes from the tile's first value to this lane's first chunk
    int lane_at;           // its index of the sum in the tile, where that lies along memory
    uint32_t address[ADDRESSES];  // of this lane's reads in a half of LDS
    const char *base, *base1;  // of the tile, at the step to load; base1: of its rows in the other half of the operand's
    int64_t bytes, bytes1;     // from there to the operand's end
    int64_t left;              // of the sum

    // Row of memory, from the tile's first, of a row of an ALONG tile.  A lane's share of r and a load's have no bits in common, and go
    // through this one by one.
    static __device__ __forceinline__ int row_of(int r)
    {
        const int in = r % (NT * 32);
        if constexpr (PAIRS) return (r - in) / 2 + in % 32 * (NT / 2) + in / 64;
        return r - in + in % 32 * NT + in / 32;
    }

    __device__ __forceinline__ void begin(int64_t stride, int first_row)
    {
        const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, r = wave * EACH + lane / (64 / EACH);
        if constexpr (ALONG) {
            lane_at = ((lane % SLOTS) ^ key(r)) * VALUES;
            lane_offset = static_cast<uint32_t>(row_of(r) * static_cast<int>(stride * sizeof(T)) + lane_at * static_cast<int>(sizeof(T)));
#pragma unroll
            for (int kk = 0; kk < ADDRESSES; ++kk) {
                const int row = first_row + threadIdx.x % 32, chunk = 2 * kk + lane / 32;
                address[kk] = row * STEP + ((chunk ^ key(row)) * 16);
            }
        } else {
            lane_at = 0;
            lane_offset = static_cast<uint32_t>(r * static_cast<int>(stride * sizeof(T)) + ((lane % SLOTS) ^ key(r)) * 16);
#pragma unroll
            for (int f = 0; f < ADDRESSES; ++f) {
                const int row = first_row + f * 32;
                if constexpr (sizeof(T) == 2) {
                    const int i = threadIdx.x % 16, depth = lane / 32 * VALUES + i / 4, in = row + threadIdx.x % 32 / 16 * 16 + i % 4 * 4;
                    address[f] = depth * (ROWS * 2) + (in / VALUES ^ key(depth)) * 16 + in % VALUES * 2;
                } else {
                    // a chunk's values are of four indexes, which the key has in common
                    const int r32 = row + threadIdx.x % 32, depth = lane / 32 * VALUES;
                    address[f] = depth * (ROWS * 4) + (r32 / VALUES ^ key(depth)) * 16 + r32 % VALUES * 4;
                }
            }
        }
    }

    __device__ __forceinline__ void aim(const Operand<T> &o, int64_t row0, int64_t from)
    {
        const int64_t row_bytes = o.stride * static_cast<int64_t>(sizeof(T));
        left = o.depth - from;
        if constexpr (ALONG) {
            const int64_t end = whole_words(o.depth);  // of a row
            const int64_t rows = PAIRS ? o.rows / 2 : o.rows, first = PAIRS ? row0 / 2 : row0;
            base = reinterpret_cast<const char *>(o.at + from) + first * row_bytes;
            bytes = (rows - 1 - first) * row_bytes + end - from * static_cast<int64_t>(sizeof(T));
            if constexpr (PAIRS) {
                base1 = base + rows * row_bytes;
                bytes1 = bytes;
            }
        } else {
            base = reinterpret_cast<const char *>(o.at + row0) + from * row_bytes;
            bytes = (left - 1) * row_bytes + whole_words(o.rows) - row0 * static_cast<int64_t>(sizeof(T));
        }
    }
    // Bytes of n values, in the words of 4 by which bounds are checked.
    static __device__ __forceinline__ int64_t whole_words(int64_t n) { return (n * static_cast<int64_t>(sizeof(T)) + 3) / 4 * 4; }

    // Values that the last step loaded has of the sum, where they end inside a chunk; else 0.
    __device__ __forceinline__ int torn() const { return ALONG && left < 0 && left % VALUES ? static_cast<int>(left + DEPTH) : 0; }

    // Zeros in what this lane loaded of such a step from behind the sum's end, which are other values of the operand.
    __device__ __forceinline__ void mend(char *lds, int there) const
    {
        if (lane_at >= there || lane_at + VALUES <= there) return;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            T *chunk = reinterpret_cast<T *>(lds + (j * WAVES + static_cast<int>(threadIdx.x / 64)) * 1024 + threadIdx.x % 64 * 16);
#pragma unroll
            for (int k = 1; k < VALUES; ++k)
                if (lane_at + k >= there) chunk[k] = T(0);
        }
    }

    // The step that base is at, to LDS, and on to the next one.
    __device__ __forceinline__ void load(const Operand<T> &o, char *lds)
    {
#if defined(__HIP_DEVICE_COMPILE__)  // the host's pass knows no descriptors
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        const int row_bytes = static_cast<int>(o.stride * sizeof(T));
        auto records = [](int64_t n) { return static_cast<int>(std::max<int64_t>(0, std::min<int64_t>(n, INT32_MAX))); };
        auto descriptor = [&](const char *at, int64_t n) {
            return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(at), 0, records(n), 0x00020000);  // no stride: bytes; 32-bit format
        };
        const auto all = descriptor(base, bytes);
        uint32_t offset = lane_offset;
        if constexpr (ALONG) {
            if (left < DEPTH) offset = lane_at < left ? lane_offset : 0x80000000u;  // past any end, with any row's offset too: zeros
        }
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int r = j * WAVES * EACH;  // and this wavefront's EACH rows, which are in the lane's offset
            const auto to = (LdsChunk)(lds + (j * WAVES + wave) * 1024);
            if constexpr (PAIRS) {
                // rows r + wave * EACH .. of the tile are of one half, the same one for all lanes
                const bool other = (r + wave * EACH) / 32 % 2;
                const auto half = other ? descriptor(base1, bytes1) : all;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(half, to, 16, offset + static_cast<uint32_t>(row_of(r) * row_bytes), 0, 0, 0);
            } else {
                __builtin_amdgcn_raw_ptr_buffer_load_lds(all, to, 16, offset + static_cast<uint32_t>((ALONG ? row_of(r) : r) * row_bytes), 0, 0, 0);
            }
        }
        const int64_t ahead = ALONG ? int64_t{STEP} : int64_t{DEPTH} * row_bytes;
        base += ahead;
        bytes -= ahead;
        if constexpr (PAIRS) {
            base1 += ahead;
            bytes1 -= ahead;
        }
        left -= DEPTH;
#endif
    }

    // Fragment f of 32 rows, of the kk-th 32 bytes of the sum's axis.
    __device__ __forceinline__ Chunk read(const char *lds, int f, int kk) const
    {
        if constexpr (ALONG) {
            return *reinterpret_cast<const Chunk *>(lds + address[kk] + f * 32 * STEP);
        } else if constexpr (sizeof(T) == 2) {
            Half h[2];
            h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsHalf)(lds + address[f] + kk * 2 * VALUES * ROWS * 2));
            h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsHalf)(lds + address[f] + (kk * 2 * VALUES + 4) * ROWS * 2));
            return *reinterpret_cast<Chunk *>(h);
        } else {
            Chunk p;
#pragma unroll
            for (int j = 0; j < VALUES; ++j)
                p[j] = *reinterpret_cast<const float *>(lds + address[f] + (kk * 2 * VALUES + j) * ROWS * 4);
            return p;
        }
    }
};

// The three parts of 8 float32 values: x = high + middle + low, each to nearest of what is left.
struct Parts {
    Chunk high, middle, low;

    __device__ __forceinline__ Parts(Chunk x0, Chunk x1)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a = i < 2 ? x0[i * 2] : x1[i * 2 - 4], b = i < 2 ? x0[i * 2 + 1] : x1[i * 2 - 3];
            high[i] = of_two(a, b);
            middle[i] = of_two(a, b);
            low[i] = of_two(a, b);
        }
    }

    // Two values as bfloat16 ones in a word, and what they leave in their place.
    static __device__ __forceinline__ float of_two(float &a, float &b)
    {
        using Two = __bf16 __attribute__((ext_vector_type(2)));
        using Pair = float __attribute__((ext_vector_type(2)));
        const uint32_t word = __builtin_bit_cast(uint32_t, __builtin_convertvector((Pair{a, b}), Two));
        a -= __uint_as_float(word << 16);
        b -= __uint_as_float(word & 0xFFFF0000u);
        return __uint_as_float(word);
    }
};

// The products of a workgroup's tiles, one after the other; PAIRS: their columns are those of two halves of B's rows (column0 counts both).  next() aims at the next tile to load (aim), or does nothing where there is none.
template <class T, class S, bool A_ALONG, bool B_ALONG, bool PAIRS = false>
struct Flow {
    using A = FlowTile<T, A_ALONG, S::M, S::THREADS, 1, false, S::MT>;
    using B = FlowTile<T, B_ALONG, S::N, S::THREADS, S::NEXT || PAIRS ? S::NT : 1, PAIRS, S::NT>;
    static_assert(B_ALONG || !(S::NEXT || PAIRS), "rows of a tile that lies across stay in order");
    static_assert(!PAIRS || S::NT % 2 == 0, "a wavefront's columns are as many of each half");
    static constexpr int STAGE = A::BYTES + B::BYTES;  // of LDS, which holds two
    static constexpr int GROUP = sizeof(T) == 4 ? 2 : 1;  // times 32 bytes of the sum's axis that go to the matrix core at once
    static constexpr int GROUPS = STEP / 32 / GROUP, DEPTH = A::DEPTH;
    static_assert(GROUPS % 2 == 0, "a step begins in the same registers");

    // Where A lies along memory B's loads go a group after A's, not all at once: bfloat16, 16,384 x 1024 x 8192 with B across 256 us and 251, 8192 x 2048 x
    // 2048 62.4 and 60.7; both across, 8192 x 2048 x 8192, 221 and 225.
    static constexpr bool LATE = sizeof(T) == 2 && A_ALONG;

    const Operand<T> &a, &b;
    char *lds;
    A ta;
    B tb;
    int steps = 0;  // left to load of the tile that is aimed at
    int stage = 0;  // where the step is that the matrix core is at
    int late = -1;  // where B's tile of the step goes whose loads have begun; -1: they are all on their way
    Chunk x[2][GROUP][S::MT], y[2][GROUP][S::NT];

    __device__ __forceinline__ Flow(const Operand<T> &a_, const Operand<T> &b_, char *lds_) : a(a_), b(b_), lds(lds_)
    {
        ta.begin(a.stride, S::wave_m() * (S::MT * 32));
        tb.begin(b.stride, S::wave_n() * (S::NT * 32));
    }

    static __device__ __forceinline__ int steps_of(int64_t from, int64_t to) { return static_cast<int>((to - from + DEPTH - 1) / DEPTH); }

    // A tile whose sum goes over [from, to).
    __device__ __forceinline__ void aim(int64_t row0, int64_t column0, int64_t from, int64_t to)
    {
        steps = steps_of(from, to);
        ta.aim(a, row0, from);
        tb.aim(b, column0, from);
    }

    template <class Next>
    __device__ __forceinline__ void load(int to, Next next)
    {
        if (steps == 0) next();
        if (steps == 0) return;
        ta.load(a, lds + to * STAGE);
        late = to;
        if constexpr (!LATE) load_late();
        --steps;
    }

    __device__ __forceinline__ void load_late()
    {
        if (late < 0) return;
        tb.load(b, lds + late * STAGE + A::BYTES);
        late = -1;
    }

    // Once the loads of stage `s`, a tile's last ones and those of ta and tb before now, are there.
    __device__ __forceinline__ void mend(int s) const
    {
        if (ta.torn()) ta.mend(lds + s * STAGE, ta.torn());
        if (tb.torn()) tb.mend(lds + s * STAGE + A::BYTES, tb.torn());
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }

    __device__ __forceinline__ void read(int g)
    {
        const char *at = lds + stage * STAGE;
#pragma unroll
        for (int k = 0; k < GROUP; ++k) {
#pragma unroll
            for (int mt = 0; mt < S::MT; ++mt) x[g % 2][k][mt] = ta.read(at, mt, g * GROUP + k);
#pragma unroll
            for (int nt = 0; nt < S::NT; ++nt) y[g % 2][k][nt] = tb.read(at + A::BYTES, nt, g * GROUP + k);
        }
    }

    __device__ __forceinline__ void multiply_group(Acc (&c)[S::MT][S::NT], int g)
    {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
                for (int nt = 0; nt < S::NT; ++nt) multiply(x[g % 2][0][mt], y[g % 2][0][nt], c[mt][nt], bf16());
        } else {
            Chunk high[S::NT], middle[S::NT], low[S::NT];
#pragma unroll
            for (int nt = 0; nt < S::NT; ++nt) {
                const Parts p(y[g % 2][0][nt], y[g % 2][1][nt]);
                high[nt] = p.high, middle[nt] = p.middle, low[nt] = p.low;
            }
#pragma unroll
            for (int mt = 0; mt < S::MT; ++mt) {
                const Parts p(x[g % 2][0][mt], x[g % 2][1][mt]);
                auto add = [&](const Chunk &a, const Chunk (&b)[S::NT]) {
#pragma unroll
                    for (int nt = 0; nt < S::NT; ++nt) multiply(a, b[nt], c[mt][nt], bf16());
                };
                add(p.low, high);
                add(p.high, low);
                add(p.middle, middle);
                add(p.middle, high);
                add(p.high, middle);
                add(p.high, high);
            }
        }
    }

    // float32 sums that are not finite, by float32 instructions, straight from memory.  Others stay as they are, whatever is in other rows.
    __device__ __forceinline__ void again(Acc (&c)[S::MT][S::NT], int64_t row0, int64_t column0, int64_t from, int64_t to) const
    {
        if constexpr (sizeof(T) == 4) {
            // Those of rows and columns that are not there, and may hold anything, do not count.
            const int64_t columns = PAIRS ? b.rows / 2 : b.rows, column1 = PAIRS ? column0 / 2 : column0;
            const int rows = static_cast<int>(std::min<int64_t>(S::M, a.rows - row0)) - S::row(0, 0);
            float none = 0;  // or NaN
#pragma unroll
            for (int nt = 0; nt < S::NT; ++nt) {
                const int across = PAIRS ? S::wave_n() * (S::NT * 16) + threadIdx.x % 32 * (S::NT / 2) + nt / 2 : S::column(nt);
                const bool there = column1 + across < columns;
#pragma unroll
                for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) none = there && mt * 32 + i / 4 * 8 + i % 4 < rows ? fmaf(c[mt][nt][i], 0.0f, none) : none;
            }
            if (!__any(none != none)) return;
            const int lane = threadIdx.x % 32, later = threadIdx.x % 64 / 32;
            const T *pb[S::NT];
#pragma unroll
            for (int nt = 0; nt < S::NT; ++nt) {
                const int64_t wave0 = S::wave_n() * (S::NT * 32);
                int64_t row;
                if constexpr (PAIRS) row = nt % 2 * (b.rows / 2) + std::min<int64_t>((column0 + wave0) / 2 + lane * (S::NT / 2) + nt / 2, b.rows / 2 - 1);
                else row = std::min<int64_t>(column0 + wave0 + (S::NEXT ? lane * S::NT + nt : nt * 32 + lane), b.rows - 1);
                pb[nt] = b.at + row * (B_ALONG ? b.stride : 1);
            }
#pragma unroll
            for (int mt = 0; mt < S::MT; ++mt) {
                const int64_t row = std::min<int64_t>(row0 + S::wave_m() * (S::MT * 32) + mt * 32 + lane, a.rows - 1);
                const T *pa = a.at + row * (A_ALONG ? a.stride : 1);
                Acc d[S::NT];
#pragma unroll
                for (int nt = 0; nt < S::NT; ++nt) d[nt] = Acc{};
                for (int64_t k0 = from; k0 < to; k0 += 2) {
                    const int64_t k = k0 + later;
                    const float u = k < to ? pa[k * (A_ALONG ? 1 : a.stride)] : 0.0f;
#pragma unroll
                    for (int nt = 0; nt < S::NT; ++nt)
                        d[nt] = __builtin_amdgcn_mfma_f32_32x32x2f32(u, k < to ? pb[nt][k * (B_ALONG ? 1 : b.stride)] : 0.0f, d[nt], 0, 0, 0);
                }
#pragma unroll
                for (int nt = 0; nt < S::NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) c[mt][nt][i] = fabsf(c[mt][nt][i]) < INFINITY ? c[mt][nt][i] : d[nt][i];
            }
        }
    }

    // The next stage is there, for all wavefronts, and nobody reads what they have read any more.
    __device__ __forceinline__ void meet()
    {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        if (steps == 0) mend(stage ^ 1);  // a tile's last step was loaded last
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }

    // Once, before the first tile.
    template <class Next>
    __device__ __forceinline__ void begin(Next next)
    {
        load(0, next);
        load_late();
        const int torn_a = ta.torn(), torn_b = tb.torn();
        load(1, next);
        load_late();
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (torn_a) ta.mend(lds, torn_a);
        if (torn_b) tb.mend(lds + A::BYTES, torn_b);
        if (steps == 0) mend(1);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        read(0);
    }

    // The next tile's sum, of `count` steps, into c.
    template <class Next>
    __device__ __forceinline__ void run(Acc (&c)[S::MT][S::NT], int count, Next next)
    {
#pragma unroll
        for (int mt = 0; mt < S::MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < S::NT; ++nt) c[mt][nt] = Acc{};
        for (; count > 0; --count) {
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                if (g + 1 < GROUPS) {
                    if (LATE && g == 0) load_late();
                    read(g + 1);
                } else {
                    meet();
                    load(stage, next);
                    stage ^= 1;
                    read(0);
                }
                multiply_group(c, g);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        load_late();  // before the tile's end
    }
};

}  // namespace
}  // namespace head_impl
