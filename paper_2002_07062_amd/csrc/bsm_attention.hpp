// Device code shared by the attention kernels: operand tiles in LDS, matrix-core fragments of
// them, and the online softmax of a wave's 32 query rows.
//
// Every kernel keeps one row of the result per lane.  v_mfma_f32_32x32x16_bf16 returns, in lane
// (li, h) = (lane & 31, lane >> 5), column li and rows 8 (i / 4) + 4 h + i % 4, i = 0..15.  So the
// transposed scores S^T = K Q^T give each lane one query (column li) and 16 of 32 keys: the row
// maximum and sum are taken in the lane, with one exchange between lanes l and l + 32, and the
// factors that rescale a row are one register.  Its registers are also the second operand of the
// next product, O^T = V^T P^T, without any exchange: an operand lane holds 8 values of the
// reduction axis, and which 8 keys those are is free as long as both operands agree.  They are
// the keys 4 h + {0..3} and 8 + 4 h + {0..3} of a block of 16, which registers 8 s .. 8 s + 7 of
// the scores hold.  V^T's lanes read the same keys of one column with ds_read_b64_tr_b16.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "bsm_attention_launch.hpp"

namespace bsm_att {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
// 16-byte accesses at any element boundary
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kWave = 64;
constexpr int kRows = 32;  // rows of the result per wave
constexpr float kInf = __builtin_huge_valf();
constexpr int kAhead = 3;      // fragments read ahead of their use (of 1 .. 6 the fastest; with more, dq spills more registers)
constexpr int kMayCross = 0x6; // of the fixed order: vector and scalar arithmetic may move

// ------------------------------------------------------------------------------- LDS tiles
// A tile is ROWS x D bf16, row after row, in 16-byte chunks whose place in the row is permuted
// (an exclusive or with bits of the row).  Fragments are read two ways: 16 consecutive rows at one
// chunk (row_frag), and 4 consecutive rows at 4 neighbouring chunks (col_frag); with these bits
// both touch every one of the 64 banks once per 256 bytes.
// D: head dimensions up to it, 64, 96 or 128; a row of 96 takes the place of one of 128.
template <int D>
struct Tile {
    static_assert(D == 64 || D == 96 || D == 128, "head dimensions are padded to 64, 96 or 128");
    static constexpr int kChunks = D == 64 ? 8 : 16;
    static constexpr int kPitch = 8 * kChunks;       // elements
    static constexpr int kRowBytes = 2 * kPitch;
    __device__ static __forceinline__ int place(int row, int chunk) {
        const int f = D == 64 ? (((row >> 1) & 1) << 2) | ((row >> 2) & 3) : ((row & 3) << 2) | ((row >> 2) & 3);
        return row * kChunks + (chunk ^ f);
    }
};

// Where a lane's fragments lie, in bytes from the start of a tile: the same for every 16 rows, so that what
// changes from read to read is a constant of the instruction.  `base`: bytes added to all of them.
template <int D>
struct RowFrags {
    int at[D / 16];
    __device__ __forceinline__ explicit RowFrags(int lane, int base = 0) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) at[i] = base + 16 * Tile<D>::place(lane & 31, 2 * i + (lane >> 5));
    }
    // lane (li, h): elements 16 s + 8 h .. + 7 of row r0 + li; r0 a multiple of 16
    __device__ __forceinline__ bf16x8 read(const uint16_t* lds, int r0, int s) const {
        return *reinterpret_cast<const bf16x8*>(reinterpret_cast<const char*>(lds) + at[s] + r0 * Tile<D>::kRowBytes);
    }
};
// Column blocks t0 .. t0 + TILES - 1 of 32.
template <int D, int TILES = D / 32>
struct ColFrags {
    int at[2][TILES];
    __device__ __forceinline__ explicit ColFrags(int lane, int t0 = 0, int base = 0) {
        const int g = lane >> 4, s = lane & 15;
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const int r = 4 * (g >> 1) + (s >> 2), c = 32 * (t0 + t) + 16 * (g & 1) + 4 * (s & 3);
            at[0][t] = base + 16 * Tile<D>::place(r, c >> 3) + 2 * (c & 7);
            at[1][t] = base + 16 * Tile<D>::place(r + 8, c >> 3) + 2 * (c & 7);
        }
    }
    // lane (li, h): column 32 (t0 + t) + li of rows r0 + 4 h + {0..3} and r0 + 8 + 4 h + {0..3}; r0 a
    // multiple of 16.  ds_read_b64_tr_b16 works in groups of 16 lanes: lane s points at row s / 4,
    // columns 4 (s % 4) .. + 3 of a 4 x 16 block and receives the block's column s.
    __device__ __forceinline__ bf16x8 read(const uint16_t* lds, int r0, int t) const {
        const char* p = reinterpret_cast<const char*>(lds) + r0 * Tile<D>::kRowBytes;
        union {
            i16x4 half[2];
            bf16x8 all;
        } u;
        u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + at[0][t]));
        u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + at[1][t]));
        return u.all;
    }
};

// Where rows and chunks that do not exist are read: a load that is always done, from one place or the
// other, stays in flight; one inside a branch is waited for at the branch's end.
static __device__ __attribute__((aligned(16))) const uint16_t kZeros[128] = {};
// (Through the address space of device memory: a pointer chosen between two would be read by flat loads,
// which also wait in line with LDS.)
__device__ __forceinline__ u32x4 load_global(const uint16_t* p) {
    return *(const __attribute__((address_space(1))) u32x4_any*)(p);
}
__device__ __forceinline__ u32x4 load_or_zero(const uint16_t* p, bool live) { return load_global(live ? p : kZeros); }

// Carries a ROWS x D tile from memory to LDS, 16 bytes at a time: `begin` starts the loads of the tile
// whose first row is at p and of which rows lo .. hi - 1 exist, `end` leaves them in LDS; then a
// tile_barrier makes them visible.  Rows and chunks that do not exist are zeros (a masked
// probability times what lies there must be zero).
// DIRECT: memory to LDS without registers on the way, which takes 16-byte aligned pieces.  The place of a
// lane's 16 bytes in LDS is fixed (64 lanes side by side), so the lane reads the chunk that belongs there.
template <int D, int ROWS, int THREADS, bool DIRECT>
struct Stage {
    static constexpr int kN = ROWS * Tile<D>::kChunks / THREADS;
    static_assert(kN >= 1 && ROWS * Tile<D>::kChunks % THREADS == 0, "");
    u32x4 r[DIRECT ? 1 : kN];
    uint32_t off[DIRECT ? kN : 1];  // bytes from the tile's first row, for whole tiles
    bool near;                      // the offsets fit
    bool live;                      // the thread's chunks exist (they have the same number in all its rows)
    __device__ static __forceinline__ int row(int tid, int j) { return (tid + THREADS * j) / Tile<D>::kChunks; }
    __device__ static __forceinline__ int chunk(int tid, int j) {
        const int c = tid % Tile<D>::kChunks;
        return DIRECT ? Tile<D>::place(row(tid, j), c) % Tile<D>::kChunks : c;
    }
    // `stride` of the rows of all the tiles to come
    __device__ __forceinline__ void init(int tid, int64_t stride, int chunks) {
        if constexpr (DIRECT) {
            static_assert(THREADS / Tile<D>::kChunks % 16 == 0, "a thread's chunk is the same in all its rows");
            near = stride < (int64_t{1} << 24);
            live = chunk(tid, 0) < chunks;
#pragma unroll
            for (int j = 0; j < kN; ++j) off[j] = static_cast<uint32_t>(2 * (row(tid, j) * stride + 8 * chunk(tid, j)));
        }
    }
    __device__ __forceinline__ void piece(int tid, int j, uint16_t* lds, const uint16_t* p, bool live) {
        const uint16_t* from = live ? p : kZeros;
        if constexpr (DIRECT) {
            uint16_t* to = lds + 8 * (64 * __builtin_amdgcn_readfirstlane(tid >> 6) + THREADS * j);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                             (__attribute__((address_space(3))) void*)to, 16, 0, 0);
        } else {
            r[j] = load_global(from);
        }
    }
    __device__ __forceinline__ void begin(int tid, uint16_t* lds, const uint16_t* p, int64_t stride, int lo, int hi, int chunks) {
        if constexpr (DIRECT) {
            if (near && lo <= 0 && hi >= ROWS) {  // no row to leave out: one base, offsets as they are
                if (!live) return;                // (the chunk is zero since clear_tiles)
#pragma unroll
                for (int j = 0; j < kN; ++j)
                    __builtin_amdgcn_global_load_lds(
                        (const __attribute__((address_space(1))) void*)(reinterpret_cast<const char*>(p) + off[j]),
                        (__attribute__((address_space(3))) void*)(lds + 8 * (64 * __builtin_amdgcn_readfirstlane(tid >> 6) + THREADS * j)),
                        16, 0, 0);
                return;
            }
        }
#pragma unroll
        for (int j = 0; j < kN; ++j) {
            const int i = row(tid, j), c = chunk(tid, j);
            piece(tid, j, lds, p + i * stride + 8 * c, i >= lo && i < hi && c < chunks);
        }
    }
    __device__ __forceinline__ void end(int tid, uint16_t* lds) const {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int j = 0; j < kN; ++j) *reinterpret_cast<u32x4*>(lds + 8 * Tile<D>::place(row(tid, j), chunk(tid, j))) = r[j];
        }
    }
};

// Zeros in the chunks of all tiles that no load of a whole tile touches, where the head dimension ends short
// of D.
template <int D, bool DIRECT>
__device__ __forceinline__ void clear_tiles(uint16_t* tiles, int elems, int tid, int threads, int chunks) {
    if (DIRECT && chunks < D / 8) {
        for (int i = 8 * tid; i < elems; i += 8 * threads) *reinterpret_cast<u32x4*>(tiles + i) = u32x4{0, 0, 0, 0};
        __syncthreads();
    }
}

// The second operand of a product whose columns are 32 rows of a matrix in memory: lane (li, h)
// holds elements 16 step + 8 h .. + 7 of its row; zero where the row does not exist.
template <int D>
struct RowOperand {
    bf16x8 f[D / 16];
    __device__ __forceinline__ void load(const uint16_t* row, bool live, int h, int chunks) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            f[s] = __builtin_bit_cast(bf16x8, load_or_zero(row + 8 * (2 * s + h), live && 2 * s + h < chunks));
        }
    }
};

__device__ __forceinline__ f32x16 zero16() {
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = 0.0f;
    return z;
}

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Runs use(i, fragment i), i = 0 .. N - 1, with the next AHEAD fragments already on their way from LDS.
// The order is held as it is written: left alone, the compiler moves each read to right before its use,
// and every matrix instruction then waits for LDS.
template <int N, int AHEAD, class Read, class Use>
__device__ __forceinline__ void pipelined(Read read, Use use) {
    bf16x8 f[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD && i < N; ++i) f[i] = read(i);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bf16x8 now = f[i % AHEAD];
        if (i + AHEAD < N) f[i % AHEAD] = read(i + AHEAD);
        __builtin_amdgcn_sched_barrier(kMayCross);
        use(i, now);
        __builtin_amdgcn_sched_barrier(kMayCross);
    }
}

// 32 KT rows of the tile (from row r0) times the operand's 32 rows: lane (li, h) gets column li
// (operand row) and, in acc[k], tile rows r0 + 32 k + 8 (i / 4) + 4 h + i % 4.
template <int D, int KT>
__device__ __forceinline__ void row_product(f32x16 (&acc)[KT], const RowFrags<D>& at, const uint16_t* lds, int r0, const RowOperand<D>& q) {
    constexpr int kSteps = D / 16;
#pragma unroll
    for (int k = 0; k < KT; ++k) acc[k] = zero16();
    pipelined<KT * kSteps, kAhead>(
        [&](int i) { return at.read(lds, r0 + 32 * (i / kSteps), i % kSteps); },
        [&](int i, bf16x8 a) { acc[i / kSteps] = mfma(a, q.f[i % kSteps], acc[i / kSteps]); });
}

// Blocks of 32 x 32 as operands of 16 rows, rounded to bf16 (nearest even): probabilities and score
// gradients are rounded once, as operands of the next product, whose sums stay in fp32.
template <int KT>
__device__ __forceinline__ void to_operands(bf16x8 (&b)[2 * KT], const f32x16 (&x)[KT]) {
#pragma unroll
    for (int s = 0; s < 2 * KT; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) b[s][e] = static_cast<__bf16>(x[s / 2][8 * (s % 2) + e]);
}

// acc[t] += (columns of block t of tile rows r0 .. r0 + 16 N - 1)^T times N operands of 16 rows each: lane li
// keeps its column of them, rows 8 (i / 4) + 4 h + i % 4 of the block's columns.
template <int D, int TILES, int N>
__device__ __forceinline__ void col_product(f32x16 (&acc)[TILES], const ColFrags<D, TILES>& at, const uint16_t* lds, int r0,
                                            const bf16x8 (&b)[N]) {
    pipelined<N * TILES, kAhead>([&](int i) { return at.read(lds, r0 + 16 * (i / TILES), i % TILES); },
                                 [&](int i, bf16x8 a) { acc[i % TILES] = mfma(a, b[i / TILES], acc[i % TILES]); });
}

// f(v of lane l, v of lane l ^ 32), the same in both: v_permlane32_swap exchanges the upper half of one
// register with the lower half of another.  Written out because the compiler, given the builtin with two
// copies of one value, uses one of its two results twice; the s_nop is the distance that the
// instruction keeps from the one that wrote its operand.
template <class F>
__device__ __forceinline__ float both_halves(float v, F f) {
    float x = v, y = v;
    asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(x), "+v"(y));
    return f(x, y);
}
__device__ __forceinline__ float half_sum(float v) {
    return both_halves(v, [](float x, float y) { return x + y; });
}
__device__ __forceinline__ float half_max(float v) {
    return both_halves(v, [](float x, float y) { return fmaxf(x, y); });
}

// Index along the tile's rows of register i in half h.
__device__ __forceinline__ constexpr int reg_row(int i) { return 8 * (i >> 2) + (i & 3); }

// Columns 32 t .. 32 t + 31 of lane li's row of the result, f * acc, as bf16 (nearest even): the two
// halves of a wave exchange 4-element groups so that each stores 16 bytes.
__device__ __forceinline__ void store_block(uint16_t* row, bool live, const f32x16& acc, float f, int t, int h, int chunks) {
#pragma unroll
    for (int g = 0; g < 4; g += 2) {
        unsigned int a[2], b[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const bf16x2 va = {static_cast<__bf16>(f * acc[4 * g + 2 * e]), static_cast<__bf16>(f * acc[4 * g + 2 * e + 1])};
            const bf16x2 vb = {static_cast<__bf16>(f * acc[4 * g + 4 + 2 * e]), static_cast<__bf16>(f * acc[4 * g + 5 + 2 * e])};
            a[e] = __builtin_bit_cast(unsigned int, va);
            b[e] = __builtin_bit_cast(unsigned int, vb);
        }
        const auto p0 = __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false);
        const auto p1 = __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false);
        const int c = 4 * t + g + h;
        const u32x4 v = {p0[0], p1[0], p0[1], p1[1]};
        if (live && c < chunks) *reinterpret_cast<u32x4_any*>(row + 8 * c) = v;
    }
}
template <int D>
__device__ __forceinline__ void store_row(uint16_t* row, bool live, const f32x16 (&acc)[D / 32], float f, int h, int chunks) {
#pragma unroll
    for (int t = 0; t < D / 32; ++t) store_block(row, live, acc[t], f, t, h, chunks);
}

// Barrier that orders the workgroup's LDS accesses and leaves loads from memory in flight.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}
// Barrier after which the tiles that were begun and ended before it are visible to the workgroup, and no
// wave reads the ones before.  What is still on its way straight to LDS is waited for.
template <bool DIRECT>
__device__ __forceinline__ void tile_barrier() {
    if constexpr (DIRECT) __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    lds_barrier();
}

// Runs step(x, buffer) for x = begin, begin + by, ..., the buffers 0 and 1 in turn and known to the compiler.
template <class Step>
__device__ __forceinline__ void in_turn(int64_t begin, int64_t end, int by, Step step) {
    for (int64_t x = begin; x < end; x += 2 * by) {
        step(x, std::integral_constant<int, 0>{});
        if (x + by < end) step(x + by, std::integral_constant<int, 1>{});
    }
}

// ------------------------------------------------------------------------- online softmax
// One pass over the keys for 32 query rows, row li in lanes li and li + 32: m is the reference
// that the exponents of a row are taken from, in log2 units of the scaled scores, l the lane's
// part of the row's sum, o the unnormalised output.  m is the row's maximum when it was last
// moved; it moves when a tile exceeds it by more than kSlack (then l and o are rescaled), so
// that probabilities stay below 2^kSlack, which neither l nor o in fp32 nor the rounding of P to
// bf16, which is relative, minds.
constexpr float kSlack = 8.0f;

template <int D>
struct Online {
    f32x16 o[D / 32];
    float m, l;

    __device__ __forceinline__ void init() {
#pragma unroll
        for (int t = 0; t < D / 32; ++t) o[t] = zero16();
        m = -kInf;
        l = 0.0f;
    }
    // Takes KT blocks of 32 keys whose raw scores are s (column li, this half's 16 keys of each
    // block, -inf where masked); c = scale * log2(e) > 0.  s becomes the probabilities.
    template <int KT>
    __device__ __forceinline__ void weigh(f32x16 (&s)[KT], float c) {
        float top = s[0][0];
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[k][i]);
        top = half_max(top) * c;
        // (also where m is still -inf; a NaN leaves m as it is and reaches l below)
        if (__any(top > m + kSlack)) {
            const float next = fmaxf(m, top);
            const float f = next == -kInf ? 1.0f : __builtin_amdgcn_exp2f(m - next);
            m = next;
            l *= f;
#pragma unroll
            for (int t = 0; t < D / 32; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[t][i] *= f;
        }
        const float ref = m == -kInf ? 0.0f : m;
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[k][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k][i], c, -ref));
                sum += s[k][i];
            }
        l += sum;
    }
    __device__ __forceinline__ float row_sum() const { return half_sum(l); }
    // natural-log statistic of a row with sum `total`
    __device__ __forceinline__ float statistic(float total) const {
        return total == 0.0f ? -kInf : (m + __builtin_amdgcn_logf(total)) * kLn2;
    }
};

// Scores of keys that the row does not see become -inf: `first` is the key of register 0 in half 0
// of the block, keys lo .. hi are seen.
__device__ __forceinline__ void mask_block(f32x16& s, int first, int h, int lo, int hi) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int j = first + 4 * h + reg_row(i);
        s[i] = j >= lo && j <= hi ? s[i] : -kInf;
    }
}

}  // namespace bsm_att
