// Attention of ragged sequences in one pass over the keys, and its gradient, which forms the
// probabilities again from the saved log-sum-exp of every row.
#include <type_traits>

#include "bsm_attention.hpp"

namespace bsm_att {
namespace {

constexpr int kThreads = 256;
constexpr int kKeys = 64;  // keys (or query rows, for dk and dv) per step

__device__ __forceinline__ const uint16_t* at(const Heads& t, const Unit& u, int64_t start, int head) {
    return t.p + u.seq * t.seq + start * t.row + head * t.head;
}

// The keys that query row i of a sequence sees are lo .. hi.
struct Seen {
    int lo, hi;
};
__device__ __forceinline__ Seen seen_keys(int i, int q_len, int kv_len, Mask m) {
    Seen s = {0, kv_len - 1};
    if (m.causal) {
        const int p = i + kv_len - q_len;
        s.hi = p < s.hi ? p : s.hi;
        if (m.window > 0 && p - m.window + 1 > 0) s.lo = p - m.window + 1;  // (of at most kMostRows each, which fits)
    }
    return s;
}

// Where two waves that share query rows hand over sums and statistics, one lane's: word n at n * kWave.
template <int D>
__device__ __forceinline__ float* exchange(void* lds, int pair, int lane) {
    static_assert(2 * (D / 2 + 2) * kWave * 4 <= 4 * kKeys * 2 * Tile<D>::kPitch, "two pairs within the tiles");
    return static_cast<float*>(lds) + pair * (D / 2 + 2) * kWave + lane;
}
template <int TILES, class F>
__device__ __forceinline__ void each_sum(f32x16 (&acc)[TILES], F f) {
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            float v = acc[t][e];
            f(16 * t + e, v);
            acc[t][e] = v;
        }
}

// ------------------------------------------------------------------------------------ forward
// o_i = sum_j exp(s_ij - lse_i) v_j in one pass over the keys (see Online): each wave keeps 32 query rows, its
// operand of the scores, their output and statistics in registers, and the workgroup brings 64 keys and
// values at a time through LDS, the next ones on their way meanwhile.  Two workgroups share a CU.  Whole
// blocks that the mask hides are left out, and blocks that it does not touch are not masked.
// KS = 1: four waves of 32 rows.  KS = 2: 64 rows, two waves of each 32 with half of every step's keys, joined
// at the end; for plans whose longest units would outlast the others (see query_rows).  STEP: keys of a step;
// 128 where few_units, as a wave alone on its SIMD takes 64 keys as fast as it takes 32, but would keep a third
// workgroup off the CU (heads of 64, us with 64 and 128: 2 x 512 rows, 12 heads 8.9, 7.6; 4096, 8 heads, causal
// 46.7, 37.5; 8 x 512, 12 heads, 768 units 11.3, 13.5; longer heads no faster).
// Bound by the matrix cores with the exponentials between them, and on random data by the power that both
// take: 4 x 4096 causal rows, 32/8 heads of 128, 570 .. 610 us = 901 .. 964 TFLOP/s with the card's clock (a
// library's 8192^3 product: 1203 .. 1221), of whose cycles the matrix cores are busy for 49% and the vector units for
// another 48%, at 1.9 .. 2.0 of 2.4 GHz; 475 us on zeros.
template <int D, bool DIRECT, int KS, int STEP>
__global__ __launch_bounds__(kThreads, 2) void attention_kernel(const SequenceArgs a, const Unit* __restrict__ units) {
    constexpr int kKeys = STEP;
    __shared__ __align__(16) uint16_t lds[2][2][kKeys * Tile<D>::kPitch];  // buffer, K or V
    const Unit u = units[blockIdx.x];
    if (u.rows <= 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, li = lane & 31, h = lane >> 5;
    const int chunks = a.dim / 8;
    constexpr int kRowWaves = kThreads / kWave / KS, kBlocks = kKeys / 32 / KS;
    const int i0 = u.first + kRows * (wave % kRowWaves), i = i0 + li;
    const int x = wave / kRowWaves;  // which of every step's keys
    const bool live = i < u.first + u.rows;
    RowOperand<D> q;
    q.load(at(a.q, u, u.q_start + i, u.head), live, h, chunks);

    const Seen mine = seen_keys(i, u.q_len, u.kv_len, a.mask);
    // keys that some row of the wave sees, that all its rows see, and that some row of the unit sees
    const int last = u.first + u.rows - 1;
    const Seen w0 = seen_keys(i0, u.q_len, u.kv_len, a.mask), w1 = seen_keys(i0 + kRows - 1, u.q_len, u.kv_len, a.mask);
    const Seen u0 = seen_keys(u.first, u.q_len, u.kv_len, a.mask), u1 = seen_keys(last, u.q_len, u.kv_len, a.mask);
    const int begin = u0.lo / kKeys * kKeys, end = u1.hi + 1;
    const bool any_row = i0 <= last;

    const uint16_t* kp = at(a.k, u, u.kv_start, u.head / a.group);
    const uint16_t* vp = at(a.v, u, u.kv_start, u.head / a.group);
    Stage<D, kKeys, kThreads, DIRECT> sk, sv;
    Online<D> st;
    st.init();
    const float c = a.scale * kLog2e;
    clear_tiles<D, DIRECT>(lds[0][0], sizeof(lds) / 2, tid, kThreads, chunks);
    sk.init(tid, a.k.row, chunks);
    sv.init(tid, a.v.row, chunks);
    if (begin < end) {
        sk.begin(tid, lds[0][0], kp + begin * a.k.row, a.k.row, 0, u.kv_len - begin, chunks);
        sv.begin(tid, lds[0][1], vp + begin * a.v.row, a.v.row, 0, u.kv_len - begin, chunks);
        sk.end(tid, lds[0][0]);
        sv.end(tid, lds[0][1]);
    }
    const int offset = x * 32 * kBlocks;
    const RowFrags<D> rows_at(lane, offset * Tile<D>::kRowBytes);
    const ColFrags<D> cols_at(lane, 0, offset * Tile<D>::kRowBytes);
    // the tiles read and the tiles written in a step are apart
    auto step = [&](int j0, uint16_t* __restrict__ next_k, uint16_t* __restrict__ next_v, const uint16_t* __restrict__ now_k,
                    const uint16_t* __restrict__ now_v) __attribute__((always_inline)) {
        tile_barrier<DIRECT>();
        const int next = j0 + kKeys;
        if (next < end) {
            sk.begin(tid, next_k, kp + next * a.k.row, a.k.row, 0, u.kv_len - next, chunks);
            sv.begin(tid, next_v, vp + next * a.v.row, a.v.row, 0, u.kv_len - next, chunks);
        }
        const int j = j0 + offset, j_end = j + 32 * kBlocks;
        if (any_row && j <= w1.hi && j_end > w0.lo) {
            f32x16 s[kBlocks];
            row_product<D>(s, rows_at, now_k, 0, q);
            if (j < w1.lo || j_end - 1 > w0.hi) {
#pragma unroll
                for (int k = 0; k < kBlocks; ++k) mask_block(s[k], j + 32 * k, h, mine.lo, mine.hi);
            }
            st.weigh(s, c);
            bf16x8 p[2 * kBlocks];
            to_operands(p, s);
            col_product(st.o, cols_at, now_v, 0, p);
        }
        if (next < end) {
            sk.end(tid, next_k);
            sv.end(tid, next_v);
        }
    };
    in_turn(begin, end, kKeys, [&](int j0, auto buf) { step(j0, lds[1 - buf][0], lds[1 - buf][1], lds[buf][0], lds[buf][1]); });
    float total = st.row_sum();
    if constexpr (KS == 2) {  // the other wave's part of the row: under the larger reference of the two
        float* other = exchange<D>(lds, wave % kRowWaves, lane);
        lds_barrier();  // the tiles are read
        if (x == 1) {
            each_sum(st.o, [&](int n, float v) { other[n * kWave] = v; });
            other[D / 2 * kWave] = st.m;
            other[(D / 2 + 1) * kWave] = total;
        }
        lds_barrier();
        if (x == 1) return;
        const float m = other[D / 2 * kWave], ref = fmaxf(st.m, m);
        const float f0 = st.m == -kInf ? 0.0f : __builtin_amdgcn_exp2f(st.m - ref), f1 = m == -kInf ? 0.0f : __builtin_amdgcn_exp2f(m - ref);
        each_sum(st.o, [&](int n, float& v) { v = f0 * v + f1 * other[n * kWave]; });
        total = f0 * total + f1 * other[(D / 2 + 1) * kWave];
        st.m = ref;
    }
    // a row that sees nothing, or only scores of -inf, is zero
    const float f = total == 0.0f ? 0.0f : 1.0f / total;
    uint16_t* out = a.o.p + u.seq * a.o.seq + (u.q_start + i) * a.o.row + u.head * a.o.head;
    store_row<D>(out, live, st.o, f, h, chunks);
    if (a.lse && live && h == 0) a.lse[u.head * a.total_q + u.lse_row + i] = st.statistic(total);
}

// ----------------------------------------------------------------------------------- backward
// A row's statistic as the reference of its exponents: rows that saw nothing get +inf, which makes
// every probability 0.
__device__ __forceinline__ float reference(float lse) { return lse == -kInf ? kInf : lse * kLog2e; }

// dq = scale * sum_j dS_ij k_j, with dS = P (dP - delta), P = exp(s - lse), dP = do . v: query rows
// stay in registers as in the forward pass, the keys stream through LDS.  Also leaves delta.  4 x 4096 causal
// rows, 32/8 heads of 128: 826 us = 998 TFLOP/s.
// KS and STEP as in the forward pass; KS = 2 of heads over 64 takes more registers than two workgroups on a CU
// have, so it is for plans that have one for each (1024 causal rows, 8 heads of 128: gradient 66.6 us with whole
// units, 54.6 so).  PARTS: some units are cut; without, the registers that it takes are free (six ragged sequences
// of 700 .. 4001, 32/8 heads of 128: gradient 875 us with it, 847 without).
template <int D, bool DIRECT, int KS, int STEP, bool PARTS>
__global__ __launch_bounds__(kThreads, D > 64 && KS == 2 ? 1 : 2) void attention_dq_kernel(const SequenceArgs a, const Unit* __restrict__ units) {
    constexpr int kKeys = STEP;
    __shared__ __align__(16) uint16_t lds[2][2][kKeys * Tile<D>::kPitch];
    const Unit u = units[blockIdx.x];
    if (u.rows <= 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, li = lane & 31, h = lane >> 5;
    const int chunks = a.dim / 8;
    constexpr int kRowWaves = kThreads / kWave / KS, kBlocks = kKeys / 32 / KS;
    const int i0 = u.first + kRows * (wave % kRowWaves), i = i0 + li;
    const int x = wave / kRowWaves;  // which of every step's keys
    const bool live = i < u.first + u.rows;
    RowOperand<D> q, dout;
    q.load(at(a.q, u, u.q_start + i, u.head), live, h, chunks);
    dout.load(at(a.dout, u, u.q_start + i, u.head), live, h, chunks);
    float delta = 0.0f, lse = -kInf;
    {
        RowOperand<D> o;
        o.load(at(a.o, u, u.q_start + i, u.head), live, h, chunks);
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                delta = __builtin_fmaf(static_cast<float>(o.f[s][e]), static_cast<float>(dout.f[s][e]), delta);
        delta = half_sum(delta);
        const int64_t r = u.head * a.total_q + u.lse_row + i;
        if (live) {
            lse = a.lse[r];
            if (h == 0 && x == 0 && (!PARTS || u.part == 0)) a.delta[r] = delta;
        }
    }
    const float ref = reference(lse);
    const Seen mine = seen_keys(i, u.q_len, u.kv_len, a.mask);
    const int last = u.first + u.rows - 1;
    const Seen w0 = seen_keys(i0, u.q_len, u.kv_len, a.mask), w1 = seen_keys(i0 + kRows - 1, u.q_len, u.kv_len, a.mask);
    const Seen u0 = seen_keys(u.first, u.q_len, u.kv_len, a.mask), u1 = seen_keys(last, u.q_len, u.kv_len, a.mask);
    int begin = u0.lo / kKeys * kKeys, end = u1.hi + 1;
    if constexpr (PARTS) {
        const int64_t steps = end > begin ? (end - begin + kKeys - 1) / kKeys : 0;
        end = min(end, begin + static_cast<int>(steps * (u.part + 1) / u.parts) * kKeys);
        begin += static_cast<int>(steps * u.part / u.parts) * kKeys;
    }
    const bool any_row = i0 <= last;
    const uint16_t* kp = at(a.k, u, u.kv_start, u.head / a.group);
    const uint16_t* vp = at(a.v, u, u.kv_start, u.head / a.group);
    Stage<D, kKeys, kThreads, DIRECT> sk, sv;
    f32x16 dq[D / 32];
#pragma unroll
    for (int t = 0; t < D / 32; ++t) dq[t] = zero16();
    const float c = a.scale * kLog2e;
    clear_tiles<D, DIRECT>(lds[0][0], sizeof(lds) / 2, tid, kThreads, chunks);
    sk.init(tid, a.k.row, chunks);
    sv.init(tid, a.v.row, chunks);
    if (begin < end) {
        sk.begin(tid, lds[0][0], kp + begin * a.k.row, a.k.row, 0, u.kv_len - begin, chunks);
        sv.begin(tid, lds[0][1], vp + begin * a.v.row, a.v.row, 0, u.kv_len - begin, chunks);
        sk.end(tid, lds[0][0]);
        sv.end(tid, lds[0][1]);
    }
    const int offset = x * 32 * kBlocks;
    const RowFrags<D> rows_at(lane, offset * Tile<D>::kRowBytes);
    const ColFrags<D> cols_at(lane, 0, offset * Tile<D>::kRowBytes);
    auto step = [&](int j0, uint16_t* __restrict__ next_k, uint16_t* __restrict__ next_v, const uint16_t* __restrict__ now_k,
                    const uint16_t* __restrict__ now_v) __attribute__((always_inline)) {
        tile_barrier<DIRECT>();
        const int next = j0 + kKeys;
        if (next < end) {
            sk.begin(tid, next_k, kp + next * a.k.row, a.k.row, 0, u.kv_len - next, chunks);
            sv.begin(tid, next_v, vp + next * a.v.row, a.v.row, 0, u.kv_len - next, chunks);
        }
        const int j = j0 + offset, j_end = j + 32 * kBlocks;
        if (any_row && j <= w1.hi && j_end > w0.lo) {
            const bool masked = j < w1.lo || j_end - 1 > w0.hi;
#pragma unroll
            for (int k = 0; k < kBlocks; ++k) {
                f32x16 s[1], dp[1];
                row_product<D>(s, rows_at, now_k, 32 * k, q);
                row_product<D>(dp, rows_at, now_v, 32 * k, dout);
                if (masked) mask_block(s[0], j + 32 * k, h, mine.lo, mine.hi);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][e], c, -ref));
                    const float ds = p * (dp[0][e] - delta);
                    // a masked score contributes nothing, whatever v holds there
                    s[0][e] = masked && s[0][e] == -kInf ? 0.0f : ds;
                }
                bf16x8 ds[2];
                to_operands(ds, s);
                col_product(dq, cols_at, now_k, 32 * k, ds);
            }
        }
        if (next < end) {
            sk.end(tid, next_k);
            sv.end(tid, next_v);
        }
    };
    in_turn(begin, end, kKeys, [&](int j0, auto buf) { step(j0, lds[1 - buf][0], lds[1 - buf][1], lds[buf][0], lds[buf][1]); });
    if constexpr (KS == 2) {
        float* other = exchange<D>(lds, wave % kRowWaves, lane);
        lds_barrier();  // the tiles are read
        if (x == 1) {
            each_sum(dq, [&](int n, float v) { other[n * kWave] = v; });
        }
        lds_barrier();
        if (x == 1) return;
        each_sum(dq, [&](int n, float& v) { v += other[n * kWave]; });
    }
    if (lse == -kInf) {  // the row saw nothing: no gradient, whatever dout holds
#pragma unroll
        for (int t = 0; t < D / 32; ++t) dq[t] = zero16();
    }
    if (PARTS && u.parts > 1) {
        if (!live) return;
        float* to = a.dq_part + (u.part_row + u.part * u.rows + i - u.first) * D + 4 * h;
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4)
                *reinterpret_cast<f32x4*>(to + 32 * t + 8 * e4) =
                    f32x4{dq[t][4 * e4], dq[t][4 * e4 + 1], dq[t][4 * e4 + 2], dq[t][4 * e4 + 3]};
        return;
    }
    uint16_t* out = a.dq.p + u.seq * a.dq.seq + (u.q_start + i) * a.dq.row + u.head * a.dq.head;
    store_row<D>(out, live, dq, a.scale, h, chunks);
}

// dv_j = sum_i P_ij do_i and dk_j = scale * sum_i dS_ij q_i over the rows of all query heads that
// share the key/value head: k, v and both sums stay in registers, the query rows stream through LDS, 64
// at a time.  No two workgroups add to one sum, so the result does not depend on timing.
// D = 64: a wave keeps 32 keys.  D = 96, 128: two waves share 32 keys (kPair): wave x of the pair forms P and
// dS for the 32 query rows of block x, the pair exchanges them through LDS as operands, and each adds up
// half of 128 columns over both blocks (of 96, wave 1 adds 32 that are not stored).  That keeps a wave's sums
// at 64 registers, so that two waves fit a SIMD and one's exponentials run beside the other's products (a wave
// that held whole sums took 400 registers and ran alone: 735 us against 475 us on six ragged causal sequences
// of 700 .. 4001 tokens, 32/8 heads of 128).  4 x 4096 causal rows, 32/8 heads of 128, 1245 .. 1287 us =
// 855 .. 884 TFLOP/s in its four products; on the six ragged ones the matrix cores are busy for 37% of the cycles, and the
// waves wait for 36% of theirs (32 x 512 rows, 12 heads of 64: 33% both).
// KS = 2, heads of 64: 64 keys, two waves of each 32 with a block of every step's query rows; for plans with little to
// do (see key_rows).
template <int D>
struct Dkv {
    static constexpr bool kPair = D > 64;
    static constexpr int kThreads = kPair ? 512 : 256;
    static constexpr int kTiles = 2;  // blocks of 32 columns that a wave adds up
};

template <int D, bool DIRECT, int KS>
__global__ __launch_bounds__(Dkv<D>::kThreads, 2) void attention_dkv_kernel(const SequenceArgs a, const Unit* __restrict__ units) {
    constexpr bool kPair = Dkv<D>::kPair;
    static_assert(KS == 1 || (KS == 2 && !kPair), "");
    constexpr int kTiles = Dkv<D>::kTiles, kBlocks = kKeys / 32;
    // (One array: of several, the compiler forgets which tiles a step reads and writes, and waits for the
    // loads on their way before every read of LDS.)
    struct Shared {
        uint16_t tile[2][2][kKeys * Tile<D>::kPitch];                             // buffer, q or dout
        float stat[2][2 * kKeys];                                   // buffer; references, then deltas
        bf16x8 exchange[kPair ? 4 : 1][kBlocks][4][kPair ? kWave : 1];  // pair, block; P and dS of 16 rows
    };
    __shared__ __align__(16) Shared lds;
    const Unit u = units[blockIdx.x];
    if (u.rows <= 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), li = lane & 31, h = lane >> 5;
    const int pair = kPair ? wave >> 1 : wave % (4 / KS), x = kPair ? wave & 1 : 0;
    const int mine_block = kPair ? x : wave / (4 / KS);  // of every step's query rows, where a wave takes one block
    const int chunks = a.dim / 8;
    const int j0 = u.first + kRows * pair, j = j0 + li;
    const bool live = j < u.first + u.rows;
    RowOperand<D> k, v;
    k.load(at(a.k, u, u.kv_start + j, u.head), live, h, chunks);
    v.load(at(a.v, u, u.kv_start + j, u.head), live, h, chunks);
    f32x16 dk[kTiles], dv[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) dk[t] = dv[t] = zero16();
    const float c = a.scale * kLog2e;
    // Query rows that see a key of the unit: i + off >= j, and i + off < j + window.  Rows before the
    // first key (`dead` of them, where there are more queries than keys) count as zeros, whatever they hold.
    const int off = u.kv_len - u.q_len;
    const int last = u.first + u.rows - 1;
    int begin = 0, end = u.q_len, dead = 0;
    if (a.mask.causal) {
        dead = max(0, -off);
        begin = max(0, u.first - off) / kKeys * kKeys;
        if (a.mask.window > 0 && static_cast<int64_t>(last) + a.mask.window - off < end) end = last + a.mask.window - off;
    }
    const int steps = end > begin ? (end - begin + kKeys - 1) / kKeys : 0;
    // the part's steps, of those of all query heads one after the other
    const int64_t all = static_cast<int64_t>(steps) * a.group, n0 = all * u.part / u.parts, total = all * (u.part + 1) / u.parts;
    const bool any_row = j0 <= last;

    Stage<D, kKeys, Dkv<D>::kThreads, DIRECT> sq, sd;
    float lse = 0.0f, delta = 0.0f;  // of row `tid` % kKeys of the step to come
    int rows_left = 0;
    clear_tiles<D, DIRECT>(lds.tile[0][0], sizeof(lds.tile) / 2, tid, Dkv<D>::kThreads, chunks);
    sq.init(tid, a.q.row, chunks);
    sd.init(tid, a.dout.row, chunks);
    auto fetch_stat = [&](int g, int r0) __attribute__((always_inline)) {
        const int64_t r = static_cast<int64_t>(u.head * a.group + g) * a.total_q + u.lse_row + min(r0 + tid % kKeys, end - 1);
        lse = a.lse[r];
        delta = a.delta[r];
        rows_left = end - r0;
    };
    auto put = [&](uint16_t* to_q, uint16_t* to_d, float* to_stat) __attribute__((always_inline)) {
        sq.end(tid, to_q);
        sd.end(tid, to_d);
        if (tid < kKeys) {
            const float ref = tid < rows_left ? reference(lse) : kInf;
            to_stat[tid] = ref;
            to_stat[kKeys + tid] = ref == kInf ? 0.0f : delta;
        }
    };
    int g = 0, r0 = begin;
    if (n0 < total) {
        g = static_cast<int>(n0 / steps);
        r0 = begin + static_cast<int>(n0 % steps) * kKeys;
        const int head = u.head * a.group + g;
        sq.begin(tid, lds.tile[0][0], at(a.q, u, u.q_start + r0, head), a.q.row, dead - r0, end - r0, chunks);
        sd.begin(tid, lds.tile[0][1], at(a.dout, u, u.q_start + r0, head), a.dout.row, dead - r0, end - r0, chunks);
        fetch_stat(g, r0);
        put(lds.tile[0][0], lds.tile[0][1], lds.stat[0]);
    }
    constexpr int kBlockBytes = 32 * Tile<D>::kRowBytes;
    const RowFrags<D> rows_at(lane, mine_block * kBlockBytes);
    const ColFrags<D, kTiles> mine_at(lane, x * kTiles, mine_block * kBlockBytes), other_at(lane, x * kTiles, (1 - x) * kBlockBytes);
    // whether the mask hides every pair of the step's query rows i0 .. i0 + 31 and the wave's keys
    auto none = [&](int i0) __attribute__((always_inline)) {
        const int p0 = i0 + off, p1 = min(i0 + 32, end) - 1 + off;  // positions
        if (!any_row || p1 < p0) return true;
        if (!a.mask.causal) return false;
        return p1 < j0 || (a.mask.window > 0 && static_cast<int64_t>(p0) - a.mask.window >= j0 + kRows - 1);
    };
    // P and dS of query rows i0 .. i0 + 31, rows `first` .. of the tiles at rows_at
    auto block = [&](int i0, int first, int first_stat, const uint16_t* now_q, const uint16_t* now_d, const float* now_stat, bf16x8 (&po)[2],
                     bf16x8 (&so)[2]) __attribute__((always_inline)) {
        f32x16 p[1], ds[1];
        row_product<D>(p, rows_at, now_q, first, k);
        row_product<D>(ds, rows_at, now_d, first, v);
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
            const f32x4 rr = *reinterpret_cast<const f32x4*>(now_stat + first_stat + 8 * e4 + 4 * h);
            const f32x4 dd = *reinterpret_cast<const f32x4*>(now_stat + kKeys + first_stat + 8 * e4 + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int y = 4 * e4 + e;
                p[0][y] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[0][y], c, -rr[e]));
                ds[0][y] = p[0][y] * (ds[0][y] - dd[e]);
            }
        }
        const int p0 = i0 + off, p1 = min(i0 + 32, end) - 1 + off;
        if (a.mask.causal && (p0 < j0 + kRows - 1 || (a.mask.window > 0 && static_cast<int64_t>(p1) - a.mask.window >= j0))) {
#pragma unroll
            for (int y = 0; y < 16; ++y) {
                const Seen s = seen_keys(i0 + 4 * h + reg_row(y), u.q_len, u.kv_len, a.mask);
                const bool sees = j >= s.lo && j <= s.hi;
                p[0][y] = sees ? p[0][y] : 0.0f;
                ds[0][y] = sees ? ds[0][y] : 0.0f;
            }
        }
        to_operands(po, p);
        to_operands(so, ds);
    };
    auto step = [&](int64_t n, uint16_t* __restrict__ next_q, uint16_t* __restrict__ next_d, float* __restrict__ next_stat,
                    const uint16_t* __restrict__ now_q, const uint16_t* __restrict__ now_d, const float* __restrict__ now_stat)
                    __attribute__((always_inline)) {
        tile_barrier<DIRECT>();
        int next_r0 = r0 + kKeys, next_g = g;
        if (next_r0 >= end) {
            next_r0 = begin;
            ++next_g;
        }
        if (n + 1 < total) {
            const int head = u.head * a.group + next_g;
            sq.begin(tid, next_q, at(a.q, u, u.q_start + next_r0, head), a.q.row, dead - next_r0, end - next_r0, chunks);
            sd.begin(tid, next_d, at(a.dout, u, u.q_start + next_r0, head), a.dout.row, dead - next_r0, end - next_r0, chunks);
            fetch_stat(next_g, next_r0);
        }
        bf16x8 po[2], so[2];
        if constexpr (kPair) {
            const bool mine = !none(r0 + 32 * x), other = !none(r0 + 32 * (1 - x));
            if (mine) {
                block(r0 + 32 * x, 0, 32 * x, now_q, now_d, now_stat, po, so);
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    lds.exchange[pair][x][s][lane] = po[s];
                    lds.exchange[pair][x][2 + s][lane] = so[s];
                }
            }
            lds_barrier();
            if (mine) {
                col_product(dv, mine_at, now_d, 0, po);
                col_product(dk, mine_at, now_q, 0, so);
            }
            if (other) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    po[s] = lds.exchange[pair][1 - x][s][lane];
                    so[s] = lds.exchange[pair][1 - x][2 + s][lane];
                }
                col_product(dv, other_at, now_d, 0, po);
                col_product(dk, other_at, now_q, 0, so);
            }
        } else if constexpr (KS == 2) {
            const int i0 = 32 * mine_block;
            if (!none(r0 + i0)) {
                block(r0 + i0, 0, i0, now_q, now_d, now_stat, po, so);
                col_product(dv, mine_at, now_d, 0, po);
                col_product(dk, mine_at, now_q, 0, so);
            }
        } else {
#pragma unroll
            for (int y = 0; y < kBlocks; ++y) {
                if (none(r0 + 32 * y)) continue;
                block(r0 + 32 * y, 32 * y, 32 * y, now_q, now_d, now_stat, po, so);
                col_product(dv, mine_at, now_d, 32 * y, po);
                col_product(dk, mine_at, now_q, 32 * y, so);
            }
        }
        if (n + 1 < total) put(next_q, next_d, next_stat);
        r0 = next_r0;
        g = next_g;
    };
    in_turn(n0, total, 1, [&](int64_t n, auto buf) {
        step(n, lds.tile[1 - buf][0], lds.tile[1 - buf][1], lds.stat[1 - buf], lds.tile[buf][0], lds.tile[buf][1], lds.stat[buf]);
    });
    if constexpr (KS == 2) {  // the other wave's sums over the same keys
        static_assert(2 * 32 * kTiles * kWave * 4 <= sizeof(lds.tile), "");
        float* other = reinterpret_cast<float*>(lds.tile) + pair * 32 * kTiles * kWave + lane;
        lds_barrier();  // the tiles are read
        if (mine_block == 1) {
            each_sum(dk, [&](int n, float y) { other[n * kWave] = y; });
            each_sum(dv, [&](int n, float y) { other[(16 * kTiles + n) * kWave] = y; });
        }
        lds_barrier();
        if (mine_block == 1) return;
        each_sum(dk, [&](int n, float& y) { y += other[n * kWave]; });
        each_sum(dv, [&](int n, float& y) { y += other[(16 * kTiles + n) * kWave]; });
    }
    if (u.parts > 1) {
        if (!live) return;
        float* to = a.part + (u.part_row + u.part * u.rows + j - u.first) * 2 * D + 4 * h;
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                const int d = 32 * (x * kTiles + t) + 8 * e4;
                if (d >= D) continue;
                *reinterpret_cast<f32x4*>(to + d) = f32x4{dk[t][4 * e4], dk[t][4 * e4 + 1], dk[t][4 * e4 + 2], dk[t][4 * e4 + 3]};
                *reinterpret_cast<f32x4*>(to + D + d) = f32x4{dv[t][4 * e4], dv[t][4 * e4 + 1], dv[t][4 * e4 + 2], dv[t][4 * e4 + 3]};
            }
        return;
    }
    const int64_t row = u.kv_start + j;
    uint16_t* to_k = a.dk.p + u.seq * a.dk.seq + row * a.dk.row + u.head * a.dk.head;
    uint16_t* to_v = a.dv.p + u.seq * a.dv.seq + row * a.dv.row + u.head * a.dv.head;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        store_block(to_k, live, dk[t], a.scale, x * kTiles + t, h, chunks);
        store_block(to_v, live, dv[t], 1.0f, x * kTiles + t, h, chunks);
    }
}

// Adds up the parts of a unit's dq, or dk and dv, in order: a thread per 8 columns of a row of one of them, and
// kJoinSlices workgroups per unit, as a few units of many parts would keep too few CUs reading (one workgroup
// each took 62 us for 32 units of 16 parts, 33 MB).  The first n_dq units are dq's.
constexpr int kJoinSlices = 8;
template <int D>
__global__ __launch_bounds__(kThreads) void attention_join_kernel(const SequenceArgs a, const Unit* __restrict__ units, int64_t n_dq) {
    const Unit u = units[blockIdx.x];
    const bool is_dq = blockIdx.x < n_dq;
    const int chunks = a.dim / 8, sums = is_dq ? 1 : 2;
    const int64_t step = static_cast<int64_t>(u.rows) * sums * D;
    for (int x = blockIdx.y * kThreads + threadIdx.x; x < sums * u.rows * chunks; x += kThreads * kJoinSlices) {
        const int c = x % chunks, sum = x / chunks % sums, j = x / chunks / sums;
        const float* from = (is_dq ? a.dq_part : a.part) + ((u.part_row + j) * sums + sum) * D + 8 * c;
        f32x4 lo = {0.0f, 0.0f, 0.0f, 0.0f}, hi = lo;
#pragma unroll 4
        for (int p = 0; p < u.parts; ++p) {
            const f32x4 y = *reinterpret_cast<const f32x4*>(from + p * step), z = *reinterpret_cast<const f32x4*>(from + p * step + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                lo[e] += y[e];
                hi[e] += z[e];
            }
        }
        const float f = sum ? 1.0f : a.scale;
        bf16x8 out;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            out[e] = static_cast<__bf16>(f * lo[e]);
            out[4 + e] = static_cast<__bf16>(f * hi[e]);
        }
        const Heads& to = is_dq ? a.dq : sum ? a.dv : a.dk;
        const int64_t row = (is_dq ? u.q_start : u.kv_start) + u.first + j;
        *reinterpret_cast<u32x4_any*>(to.p + u.seq * to.seq + row * to.row + u.head * to.head + 8 * c) = __builtin_bit_cast(u32x4, out);
    }
}

}  // namespace

// Whether 16-byte pieces of an operand lie on 16-byte boundaries.
bool aligned_pieces(const Heads& t) {
    return reinterpret_cast<uintptr_t>(t.p) % 16 == 0 && (t.seq | t.row | t.head) % 8 == 0;
}

// Calls f with D and DIRECT as constants.
template <class F>
hipError_t with_dim(int dim, bool direct, F f) {
    auto go = [&](auto d) { return direct ? f(d, std::true_type{}) : f(d, std::false_type{}); };
    switch (padded_dim(dim)) {
        case 64: return go(std::integral_constant<int, 64>{});
        case 96: return go(std::integral_constant<int, 96>{});
        default: return go(std::integral_constant<int, 128>{});
    }
}

hipError_t launch_attention(const SequenceArgs& a, const Unit* units, int64_t n, hipStream_t stream) {
    if (n == 0) return hipSuccess;
    return with_dim(a.dim, aligned_pieces(a.k) && aligned_pieces(a.v), [&](auto d, auto direct) {
        const dim3 grid(static_cast<unsigned>(n));
        if (a.unit_rows == kTileRows) return launch(attention_kernel<d(), direct(), 1, kKeys>, grid, kThreads, stream, a, units);
        if (d() == 64 && a.few_units) return launch(attention_kernel<64, direct(), 2, 2 * kKeys>, grid, kThreads, stream, a, units);
        return launch(attention_kernel<d(), direct(), 2, kKeys>, grid, kThreads, stream, a, units);
    });
}

template <int D, bool DIRECT, bool PARTS>
static hipError_t launch_dq(const SequenceArgs& a, const GradientUnits& u, hipStream_t stream) {
    const dim3 grid(static_cast<unsigned>(u.n_q));
    if (a.unit_rows == kTileRows) return launch(attention_dq_kernel<D, DIRECT, 1, kKeys, PARTS>, grid, kThreads, stream, a, u.q);
    if (D == 64 && a.few_units) return launch(attention_dq_kernel<64, DIRECT, 2, 2 * kKeys, PARTS>, grid, kThreads, stream, a, u.q);
    return launch(attention_dq_kernel<D, DIRECT, 2, kKeys, PARTS>, grid, kThreads, stream, a, u.q);
}

hipError_t launch_attention_backward(const SequenceArgs& a, const GradientUnits& u, hipStream_t stream) {
    hipError_t e = hipSuccess;
    if (u.n_q > 0)
        e = with_dim(a.dim, aligned_pieces(a.k) && aligned_pieces(a.v), [&](auto d, auto direct) {
            return u.n_q_joins > 0 ? launch_dq<d(), direct(), true>(a, u, stream) : launch_dq<d(), direct(), false>(a, u, stream);
        });
    if (e == hipSuccess && u.n_kv > 0)
        e = with_dim(a.dim, aligned_pieces(a.q) && aligned_pieces(a.dout), [&](auto d, auto direct) {
            const dim3 grid(static_cast<unsigned>(u.n_kv));
            if (d() == 64 && a.key_rows < kTileRows)
                return launch(attention_dkv_kernel<64, direct(), 2>, grid, Dkv<64>::kThreads, stream, a, u.kv);
            return launch(attention_dkv_kernel<d(), direct(), 1>, grid, Dkv<d()>::kThreads, stream, a, u.kv);
        });
    const int64_t joins = u.n_q_joins + u.n_kv_joins;
    if (e == hipSuccess && joins > 0)
        e = with_dim(a.dim, true, [&](auto d, auto) {
            return launch(attention_join_kernel<d()>, dim3(static_cast<unsigned>(joins), kJoinSlices), kThreads, stream, a, u.joins,
                          u.n_q_joins);
        });
    return e;
}

}  // namespace bsm_att
