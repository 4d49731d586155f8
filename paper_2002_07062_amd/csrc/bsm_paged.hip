// The paged key/value cache: attention of new tokens over the pages, the slots of new tokens, and
// the copy of their keys and values into the slots.
#include "bsm_attention.hpp"

namespace bsm_att {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = 4;

// Sums of tokens and pages over the requests before a thread's, and the chunk's totals.
struct Two {
    int64_t tokens, pages;
};
__device__ __forceinline__ Two scan(Two mine, Two* total, int64_t (*mem)[2]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Two x = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t t = __shfl_up(x.tokens, d, 64), p = __shfl_up(x.pages, d, 64);
        if (lane >= d) {
            x.tokens += t;
            x.pages += p;
        }
    }
    if (lane == 63) {
        mem[wave][0] = x.tokens;
        mem[wave][1] = x.pages;
    }
    __syncthreads();
    Two before = {0, 0};
    *total = {0, 0};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) {
            before.tokens += mem[w][0];
            before.pages += mem[w][1];
        }
        total->tokens += mem[w][0];
        total->pages += mem[w][1];
    }
    return {before.tokens + x.tokens - mine.tokens, before.pages + x.pages - mine.pages};
}

// ---------------------------------------------------------------------------------- attention
// One request and key/value head: the rows are (new token, query head of the group) pairs, token
// after token, so that the query heads that share a key/value head read it once.
struct Request {
    int b, head;       // request, key/value head
    int64_t q0;        // its first row in q and o
    int q_len, kv_len;
    int rows;          // q_len (at most max_q) * group; 0 where the other kernel takes the request
};

template <bool FEW>
__device__ __forceinline__ Request request(const PagedArgs& a, int64_t b, int head) {
    Request r;
    r.b = static_cast<int>(b);
    r.head = head;
    const int64_t q0 = a.q_start[r.b], q1 = a.q_start[r.b + 1];
    r.q0 = q0 < 0 ? 0 : q0 < a.tokens ? q0 : a.tokens;
    const int64_t e = q1 < r.q0 ? r.q0 : q1 < a.tokens ? q1 : a.tokens;
    r.q_len = static_cast<int>(e - r.q0);
    const int64_t most = static_cast<int64_t>(a.width) * a.cache.page_size;
    const int kv = a.kv_len[r.b];
    r.kv_len = kv < 0 ? 0 : kv < most ? kv : static_cast<int>(most);
    r.rows = min(r.q_len, a.max_q) * a.group;
    if (FEW != (r.rows <= a.few_rows)) r.rows = 0;
    return r;
}

struct Keys {
    int lo, hi;  // seen keys
};
__device__ __forceinline__ Keys seen_keys(const PagedArgs& a, const Request& r, int token) {
    const int p = token + r.kv_len - r.q_len;
    Keys k = {0, p < r.kv_len - 1 ? p : r.kv_len - 1};
    if (a.window > 0 && p - a.window + 1 > 0) k.lo = p - a.window + 1;  // (of at most kMostRows each, which fits)
    return k;
}

// Pieces of the key axis that a tile of rows needs: first .. last, each split_keys keys from
// piece * split_keys (the last one of the grid: all that is left).
struct Pieces {
    Keys keys;  // seen by some row of the tile
    int first, last;
};
__device__ __forceinline__ Pieces pieces(const PagedArgs& a, const Request& r, int r0) {
    const int r1 = min(r0 + kTileRows, r.rows) - 1;
    Pieces p;
    p.keys.lo = seen_keys(a, r, r0 / a.group).lo;
    p.keys.hi = seen_keys(a, r, r1 / a.group).hi;
    if (p.keys.hi < p.keys.lo) {
        p.first = p.last = 0;
    } else {
        p.first = min(p.keys.lo / a.split_keys, a.splits - 1);
        p.last = min(p.keys.hi / a.split_keys, a.splits - 1);
    }
    return p;
}

// Element of row `row` of the request and head in q or o.
__device__ __forceinline__ int64_t row_at(const PagedArgs& a, const Request& r, const Heads& t, int row) {
    return (r.q0 + row / a.group) * t.row + (r.head * a.group + row % a.group) * t.head;
}

// Where the part of one piece of the n-th tile (see tile_of) begins: its rows' outputs, then their references and sums.
__device__ __forceinline__ int64_t part_at(const PagedArgs& a, int D, int head, int64_t n, int piece) {
    return ((n * a.cache.heads + head) * a.splits + piece) * kTileRows * (D + 2);
}

// The n-th tile of all, of one head.  The requests follow each other, the one with the most keys first (with more than
// kThreads of them, as they come), so that the CUs end together; of each the last tiles, which see most keys, first.
// Of up to kThreads requests only the tiles that hold rows count: the others of a batch of single tokens and a few
// chunks would cost a workgroup's start each (63 single tokens and a chunk of 512, 8 kv heads: 8192 of them, 8064 empty).
// b < 0: there is none.
struct TileOf {
    int b, tile;
};
constexpr int kTileOfInts = 2 + 2 * kThreads;
__device__ __forceinline__ TileOf tile_of(const PagedArgs& a, int64_t n, int* mem) {
    if (a.batch > kThreads) return {static_cast<int>(n / a.tiles), a.tiles - 1 - static_cast<int>(n % a.tiles)};
    const int i = threadIdx.x, count = static_cast<int>(a.batch);
    int *kv = mem + 2, *tiles = kv + kThreads, mine = -1, own = 0;
    if (i < count) {
        const Request r = request<false>(a, i, 0);
        own = (r.rows + kTileRows - 1) / kTileRows;
        kv[i] = mine = r.kv_len;
        tiles[i] = own;
    }
    if (i == 0) mem[0] = -1;
    __syncthreads();
    if (own > 0) {
        int64_t before = 0;
        for (int j = 0; j < count; ++j) before += kv[j] > mine || (kv[j] == mine && j < i) ? tiles[j] : 0;
        if (n >= before && n < before + own) {
            mem[0] = i;
            mem[1] = own - 1 - static_cast<int>(n - before);
        }
    }
    __syncthreads();
    const TileOf t = {__builtin_amdgcn_readfirstlane(mem[0]), __builtin_amdgcn_readfirstlane(mem[1])};
    __syncthreads();
    return t;
}

__device__ __forceinline__ bool names_page(const PagedArgs& a, int entry) { return entry >= 0 && entry < a.cache.n_pages; }

// The rows of K and V that a thread stages: tile row i is key j0 + i of the request, the tiles follow each
// other.  Keys past its end, and keys of table entries that name no page, are zeros.  Where a key lies is carried
// on from tile to tile: a division by the page size takes as long as the exponentials of several keys.
template <int D, int ROWS, int THREADS, bool DIRECT>
struct PagedStage {
    using S = Stage<D, ROWS, THREADS, DIRECT>;
    S k, v;
    int column[S::kN], row[S::kN];  // table column of the next tile's key, and its row within the page
    int now[S::kN];                 // row of this tile's key
    int page[S::kN];  // table entries, looked at when they are used: they are loaded behind a tile's loads
    int step_columns, step_rows, last_column;
    bool near;  // strides of 32 bits
    __device__ __forceinline__ void init(const PagedArgs& a, int tid, int j0, int end) {
        step_columns = ROWS / a.cache.page_size;
        step_rows = ROWS % a.cache.page_size;
        last_column = (end - 1) / a.cache.page_size;
        near = (a.cache.page | a.cache.row) >> 32 == 0;
#pragma unroll
        for (int n = 0; n < S::kN; ++n) {
            const int j = j0 + S::row(tid, n);
            column[n] = j / a.cache.page_size;
            row[n] = j - column[n] * a.cache.page_size;
        }
    }
    // table entries of the next tile; the request has keys 0 .. end - 1
    __device__ __forceinline__ void find(const PagedArgs& a, const int32_t* table) {
#pragma unroll
        for (int n = 0; n < S::kN; ++n) {
            page[n] = table[min(column[n], last_column)];
            now[n] = row[n];
            column[n] += step_columns;
            row[n] += step_rows;
            if (row[n] >= a.cache.page_size) {
                row[n] -= a.cache.page_size;
                ++column[n];
            }
        }
    }
    __device__ __forceinline__ void begin(const PagedArgs& a, int head, int tid, int j0, int end, int chunks, uint16_t* lds_k, uint16_t* lds_v) {
#pragma unroll
        for (int n = 0; n < S::kN; ++n) {
            const int j = j0 + S::row(tid, n), c = S::chunk(tid, n);
            const bool live = j < end && names_page(a, page[n]) && c < chunks;
            int64_t from;  // (of 32-bit strides a product is one instruction)
            if (near)
                from = static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(page[n])) * static_cast<uint32_t>(a.cache.page) +
                                            static_cast<uint64_t>(static_cast<uint32_t>(now[n])) * static_cast<uint32_t>(a.cache.row));
            else
                from = page[n] * a.cache.page + now[n] * a.cache.row;
            from += head * a.cache.head + 8 * c;
            k.piece(tid, n, lds_k, a.cache.k + from, live);
            v.piece(tid, n, lds_v, a.cache.v + from, live);
        }
    }
    __device__ __forceinline__ void end(int tid, uint16_t* lds_k, uint16_t* lds_v) const {
        k.end(tid, lds_k);
        v.end(tid, lds_v);
    }
};

// Many rows (chunks of prompts): a tile has 128 rows, 32 per wave, and the waves share the staged keys, as in the
// forward pass over sequences, which bounds it too.  8 chunks of 512 over 1k .. 8k keys, 32/8 heads of 128: 289 .. 312
// us = 811 .. 876 TFLOP/s.
template <int D, bool DIRECT>
__global__ __launch_bounds__(kThreads, 2) void paged_kernel(const PagedArgs a) {
    constexpr int kKeys = 64, kTileElems = kKeys * Tile<D>::kPitch;
    // (One array: of several, the compiler forgets which tiles a step reads and writes, and waits for the
    // loads on their way before every read of LDS.)
    __shared__ __align__(16) uint16_t lds[2][2][kTileElems];  // buffer, K or V
    // A tile's pieces and heads follow each other, the heads side by side.  They are rotated from request to request: a page
    // has its heads side by side, and an XCD that only ever read one of 8 heads of 128 (workgroups go to the 8 XCDs in
    // turn) would use 2 of its 16 L2 channels, which lie 256 bytes apart.
    const int64_t n = blockIdx.x / a.cache.heads / a.splits;
    const TileOf at = tile_of(a, n, reinterpret_cast<int*>(lds));
    if (at.b < 0) return;
    const int tile = at.tile, piece = static_cast<int>(blockIdx.x / a.cache.heads % a.splits);
    const Request r = request<false>(a, at.b, static_cast<int>((blockIdx.x + at.b) % a.cache.heads));
    const int tile0 = tile * kTileRows;
    if (tile0 >= r.rows) return;
    const Pieces ps = pieces(a, r, tile0);
    if (piece < ps.first || piece > ps.last) return;

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, li = lane & 31, h = lane >> 5;
    const int chunks = a.cache.dim / 8;
    const int row0 = tile0 + kRows * wave, row = row0 + li;
    const bool live = row < r.rows;
    const bool any_row = row0 < r.rows;
    const int token = row / a.group, q_head = r.head * a.group + row % a.group;
    const int64_t q_row = r.q0 + token;
    RowOperand<D> q;
    q.load(a.q.p + q_row * a.q.row + q_head * a.q.head, live, h, chunks);
    const Keys mine = seen_keys(a, r, token);
    const Keys w0 = seen_keys(a, r, row0 / a.group), w1 = seen_keys(a, r, (row0 + kRows - 1) / a.group);

    const int from = max(ps.keys.lo, piece * a.split_keys);
    const int end = piece == a.splits - 1 ? ps.keys.hi + 1 : min(ps.keys.hi + 1, (piece + 1) * a.split_keys);
    const int begin = from / kKeys * kKeys;
    const int32_t* table = a.table + static_cast<int64_t>(r.b) * a.width;

    Online<D> st;
    st.init();
    const float c = a.scale * kLog2e;
    PagedStage<D, kKeys, kThreads, DIRECT> stage;
    if (begin < end) {
        stage.init(a, tid, begin, r.kv_len);
        stage.find(a, table);
        stage.begin(a, r.head, tid, begin, r.kv_len, chunks, lds[0][0], lds[0][1]);
        stage.find(a, table);
        stage.end(tid, lds[0][0], lds[0][1]);
    }
    const RowFrags<D> rows_at(lane);
    const ColFrags<D> cols_at(lane);
    // the tiles read and the tiles written in a step are apart
    auto step = [&](int j0, uint16_t* __restrict__ next_k, uint16_t* __restrict__ next_v, const uint16_t* __restrict__ now_k,
                    const uint16_t* __restrict__ now_v) __attribute__((always_inline)) {
        const int next = j0 + kKeys;
        tile_barrier<DIRECT>();
        if (next < end) {
            stage.begin(a, r.head, tid, next, r.kv_len, chunks, next_k, next_v);
            stage.find(a, table);
        }
        if (any_row && j0 <= w1.hi && next > w0.lo) {
            f32x16 s[kKeys / 32];
            row_product<D>(s, rows_at, now_k, 0, q);
            if (j0 < w1.lo || next - 1 > w0.hi || end < next) {
#pragma unroll
                for (int k = 0; k < kKeys / 32; ++k) mask_block(s[k], j0 + 32 * k, h, mine.lo, min(mine.hi, end - 1));
            }
            st.weigh(s, c);
            bf16x8 p[kKeys / 16];
            to_operands(p, s);
            col_product(st.o, cols_at, now_v, 0, p);
        }
        if (next < end) stage.end(tid, next_k, next_v);
    };
    in_turn(begin, end, kKeys, [&](int j0, auto buf) { step(j0, lds[1 - buf][0], lds[1 - buf][1], lds[buf][0], lds[buf][1]); });
    const float total = st.row_sum();
    if (ps.first == ps.last) {
        uint16_t* out = a.o.p + q_row * a.o.row + q_head * a.o.head;
        store_row<D>(out, live, st.o, total == 0.0f ? 0.0f : 1.0f / total, h, chunks);
    } else if (live) {
        float* part = a.tile_part + part_at(a, D, r.head, n, piece);
        float* to = part + (row - tile0) * D + 4 * h;
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<f32x4*>(to + 32 * t + 8 * g) =
                    f32x4{st.o[t][4 * g], st.o[t][4 * g + 1], st.o[t][4 * g + 2], st.o[t][4 * g + 3]};
        if (h == 0) {
            part[kTileRows * D + row - tile0] = st.m;
            part[kTileRows * (D + 1) + row - tile0] = total;
        }
    }
}

// Few rows over many keys (decode) are bound by reading the cache, so what counts is how much of it is
// in flight: the waves never wait for each other, each takes every fourth block of 32 keys and joins
// its rows with the others' at the end.  v_mfma_f32_16x16x32_bf16 keeps 16 rows (NQ times) in a quarter
// of the registers that 32 x 32 tiles take.  Its lane (n, quad) = (lane & 15, lane >> 4) returns column
// n and rows 4 quad + i, and reads 8 values of the reduction axis; as in the other kernels the scores'
// registers are the next operand: keys 4 quad + i and 16 + 4 quad + i of a block.
// A lane reads two keys' rows, n and n + 16, of K and of V.  K goes to the matrix cores as it comes; V is
// turned in LDS.  The next block's loads are issued when the scores have left K's registers.
// FULL: the head dimension is D, so that a row is read from one address or from zeros as a whole.
//
// The work is one stream: request after request, the blocks of kFewKeys keys that its rows see.  Its
// equal shares go to one workgroup for each key/value head, wherever they begin and end, so requests of
// any lengths keep all CUs busy to the end; a request whose blocks lie in several shares is joined
// afterwards.  The workgroups of a share run side by side, and with them the reads of a page's heads, which
// lie side by side too.  Each workgroup counts the stream itself, 8 bytes a request from the cache.
// 64 requests of 1k .. 32k keys, 8 kv heads of 128, 2.3 GB: 434 us = 5.3 TB/s, the joins 8 us (a plain read of as
// much: 6.0 TB/s).

// Blocks of one head of a request; one without keys has a block that writes zeros.
struct Blocks {
    Keys keys;
    int first, n;
};
__device__ __forceinline__ Blocks blocks_of(const PagedArgs& a, const Request& r) {
    Blocks x = {{0, -1}, 0, 0};
    if (r.rows == 0) return x;
    x.keys.lo = seen_keys(a, r, 0).lo;
    x.keys.hi = seen_keys(a, r, (r.rows - 1) / a.group).hi;
    x.n = 1;
    if (x.keys.hi >= x.keys.lo) {
        x.first = x.keys.lo / kFewKeys;
        x.n = x.keys.hi / kFewKeys - x.first + 1;
    }
    return x;
}

// A value that all lanes hold, as one that the compiler knows to be the same in all of them.
__device__ __forceinline__ int64_t uniform(int64_t x) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(x)), hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(x >> 32));
    return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}

// Blocks of all requests, of one head, and of those before request b.
struct Stream {
    int64_t all, before;
};
__device__ __forceinline__ Stream count_blocks(const PagedArgs& a, int64_t b, int64_t (*mem)[2]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Stream x = {0, 0};
    for (int64_t i = threadIdx.x; i < a.batch; i += kThreads) {
        const int64_t n = blocks_of(a, request<true>(a, i, 0)).n;
        x.all += n;
        if (i < b) x.before += n;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        x.all += __shfl_xor(x.all, d, 64);
        x.before += __shfl_xor(x.before, d, 64);
    }
    if (lane == 0) {
        mem[wave][0] = x.all;
        mem[wave][1] = x.before;
    }
    __syncthreads();
    x = {0, 0};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        x.all += mem[w][0];
        x.before += mem[w][1];
    }
    return {uniform(x.all), uniform(x.before)};
}
// Blocks of a share: 4 at least, else counting them and joining takes as long as reading them.  The shares go round the
// CUs evenly, one to each or two, as often as it takes for shares of up to 16: larger ones end too far apart (one round
// of equal shares of 64 requests of 1k .. 32k keys left CUs idle for 30% of the time), and a few workgroups more than
// go round keep the others waiting (64 ragged requests of up to 4096 keys, 8 kv heads of 128, 304 workgroups 100 us, 488
// 84 us; up to 8192 149, 127 us).  But there are no more than a.shares.
__device__ __forceinline__ int64_t share_of(const PagedArgs& a, int64_t blocks) {
    const int64_t even = (blocks + a.shares - 1) / a.shares, rounds = (blocks + 2 * kMostBlocks * a.round - 1) / (2 * kMostBlocks * a.round);
    int64_t share = (blocks + a.round - 1) / a.round;
    if (share > kMostBlocks) share = (blocks + 2 * rounds * a.round - 1) / (2 * rounds * a.round);
    return max(even, max(share, static_cast<int64_t>(kFewestBlocks)));
}
__device__ __forceinline__ int64_t few_part_at(const PagedArgs& a, int D, int64_t part) {
    return part * a.few_rows * (D + 2);
}

template <int D, int NQ, bool FULL>
__global__ __launch_bounds__(kThreads, 2) void paged_few_kernel(const PagedArgs a) {
    constexpr int kKeys = 32, kSteps = D / 32, kTiles = D / 16;
    static_assert(kKeys * kWaves == kFewKeys, "");
    constexpr int kRegs = NQ * kTiles * 4;  // outputs of a lane
    constexpr int kBlockBytes = kKeys * Tile<D>::kRowBytes;
    constexpr int kBytes = kWaves * (kRegs * kWave * 4 > kBlockBytes ? kRegs * kWave * 4 : kBlockBytes);
    __shared__ __align__(16) unsigned char lds[kBytes];
    __shared__ float stat[2][kWaves][16 * NQ];
    __shared__ int64_t mem[kWaves][2], s_at[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, quad = lane >> 4;
    const int chunks = a.cache.dim / 8;

    // the share: `left` blocks from block `block` of request b
    const int64_t w = blockIdx.x / a.cache.heads;
    const int head = static_cast<int>((blockIdx.x + w) % a.cache.heads);  // rotated, see paged_kernel
    int64_t b = 0, left = 0;
    int block = 0;
    if (a.shares == 0) {  // one request each
        b = w;
        left = blocks_of(a, request<true>(a, b, 0)).n;
    } else {
// (a batch of up to kThreads requests is counted and searched in one look at it)
        int64_t mine = 0, before = 0, blocks;
        if (a.batch <= kThreads) {
            if (tid < a.batch) mine = blocks_of(a, request<true>(a, tid, 0)).n;
            Two total;
            before = scan({mine, 0}, &total, mem).tokens;
            blocks = uniform(total.tokens);
        } else {
            blocks = count_blocks(a, 0, mem).all;
        }
        const int64_t share = share_of(a, blocks), start = w * share;
        left = min(share, blocks - start);
        if (left > 0) {
            if (a.batch <= kThreads) {
                if (start >= before && start < before + mine) {
                    s_at[0] = tid;
                    s_at[1] = start - before;
                }
                __syncthreads();
            }
            for (int64_t b0 = 0; a.batch > kThreads && b0 < a.batch && before <= start; b0 += kThreads) {
                mine = b0 + tid < a.batch ? blocks_of(a, request<true>(a, b0 + tid, 0)).n : 0;
                Two total;
                const int64_t at = before + scan({mine, 0}, &total, reinterpret_cast<int64_t(*)[2]>(lds)).tokens;
                if (start >= at && start < at + mine) {
                    s_at[0] = b0 + tid;
                    s_at[1] = start - at;
                }
                before = uniform(before + total.tokens);
                __syncthreads();
            }
            b = uniform(s_at[0]);
            block = static_cast<int>(uniform(s_at[1]));
        }
    }
    bool at_start = true;  // nothing of the share is done
    // The wave's V block.  A place does not depend on a multiple of 16 of the row, and chunk x ^ y lies at an
    // exclusive or of 16 y with the place of chunk x: one address each for writing and for reading.
    unsigned char* turned = lds + wave * kBlockBytes;
    int put_at = 16 * Tile<D>::place(n, quad);  // row n, chunk quad; chunk 4 e + quad is 64 e away
    // lane (n, quad): column n of rows 4 quad + {0..3} (and of those 16 further); column 16 t + n is 32 t away
    int col_at = 16 * Tile<D>::place(4 * quad + (n >> 2), (n & 3) >> 1) + 8 * (n & 1);
    const float c = a.scale * kLog2e;
    for (; left > 0; ++b, block = 0) {
        const Request r = request<true>(a, b, head);
        const Blocks bl = blocks_of(a, r);
        if (block < bl.n) {
            const int first = block, count = static_cast<int>(min(static_cast<int64_t>(bl.n - first), left));
            const bool whole = count == bl.n;
            const int64_t part_index = 2 * (w * a.cache.heads + head) + (first == 0 && !at_start ? 1 : 0);
            left -= count;
            at_start = false;
            // keys of the unit's blocks that some row sees
            const int from = (bl.first + first) * kFewKeys, end = min(bl.keys.hi + 1, from + count * kFewKeys);
            bf16x8 q[NQ][kSteps];
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
                const int row = 16 * x + n;
#pragma unroll
                for (int s = 0; s < kSteps; ++s) {
                    const uint16_t* from_q = a.q.p + row_at(a, r, a.q, row) + 8 * (4 * s + quad);
                    q[x][s] = __builtin_bit_cast(bf16x8, load_or_zero(from_q, row < r.rows && 4 * s + quad < chunks));
                }
            }
            // keys that every row sees
            const int all_lo = seen_keys(a, r, (r.rows - 1) / a.group).lo, all_hi = seen_keys(a, r, 0).hi;
            const int begin = from + wave * kKeys;
            const int32_t* table = a.table + static_cast<int64_t>(r.b) * a.width;

            f32x4 o[NQ][kTiles];
            float m[NQ], l[NQ];
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
                m[x] = -kInf;
                l[x] = 0.0f;
#pragma unroll
                for (int t = 0; t < kTiles; ++t) o[x][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            }
            u32x4 k[2][kSteps], v[2][kSteps];
            int page[2];
            auto find = [&](int j0) {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    page[y] = table[min(j0 + 16 * y + n, r.kv_len - 1) / a.cache.page_size];
                }
            };
            auto load = [&](int j0) {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int j = j0 + 16 * y + n;
                    // (keys that no row sees, as those of pages that a window has left behind, count as zeros)
                    const bool live = j >= bl.keys.lo && j <= bl.keys.hi && names_page(a, page[y]);
                    const int64_t at = page[y] * a.cache.page + (j % a.cache.page_size) * a.cache.row + r.head * a.cache.head + 8 * quad;
                    const uint16_t* kp = live ? a.cache.k + at : kZeros + 8 * quad;
                    const uint16_t* vp = live ? a.cache.v + at : kZeros + 8 * quad;
#pragma unroll
                    for (int s = 0; s < kSteps; ++s) {
                        k[y][s] = load_or_zero(kp + 32 * s, FULL || 4 * s + quad < chunks);
                        v[y][s] = load_or_zero(vp + 32 * s, FULL || 4 * s + quad < chunks);
                    }
                }
            };
            constexpr int step = kKeys * kWaves;
            if (begin < end) {
                find(begin);
                load(begin);
                find(begin + step);
            }
            for (int j0 = begin; j0 < end; j0 += step) {
                // kept as one register each, not as one for every e and t
                asm volatile("" : "+v"(put_at), "+v"(col_at));
                f32x4 s[NQ][2];
#pragma unroll
                for (int x = 0; x < NQ; ++x)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        s[x][y] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                        for (int e = 0; e < kSteps; ++e)
                            s[x][y] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[y][e]), q[x][e], s[x][y], 0, 0, 0);
                    }
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int e = 0; e < kSteps; ++e)
                        *reinterpret_cast<u32x4*>(turned + (put_at ^ 64 * e) + 16 * y * Tile<D>::kRowBytes) = v[y][e];
                const int next = j0 + step;
                if (next < end) {
                    load(next);
                    find(next + step);
                }
                // the wave's own writes, before its lanes read each other's
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup", "local");
                __builtin_amdgcn_wave_barrier();
                const bool masked = j0 < all_lo || j0 + kKeys - 1 > all_hi || j0 + kKeys > end;
#pragma unroll
                for (int x = 0; x < NQ; ++x) {
                    if (masked) {
                        const Keys mine = seen_keys(a, r, (16 * x + n) / a.group);
#pragma unroll
                        for (int y = 0; y < 2; ++y)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int j = j0 + 16 * y + 4 * quad + i;
                                s[x][y][i] = j >= mine.lo && j <= mine.hi && j < end ? s[x][y][i] : -kInf;
                            }
                    }
                    float top = s[x][0][0];
#pragma unroll
                    for (int y = 0; y < 2; ++y)
#pragma unroll
                        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[x][y][i]);
                    top = fmaxf(top, __shfl_xor(top, 16, 64));
                    top = fmaxf(top, __shfl_xor(top, 32, 64)) * c;
                    if (__any(top > m[x] + kSlack)) {
                        const float to = fmaxf(m[x], top);
                        const float f = to == -kInf ? 1.0f : __builtin_amdgcn_exp2f(m[x] - to);
                        m[x] = to;
                        l[x] *= f;
#pragma unroll
                        for (int t = 0; t < kTiles; ++t)
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[x][t][i] *= f;
                    }
                    const float ref = m[x] == -kInf ? 0.0f : m[x];
                    bf16x8 p;
#pragma unroll
                    for (int y = 0; y < 2; ++y)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][y][i], c, -ref));
                            l[x] += e;
                            p[4 * y + i] = static_cast<__bf16>(e);
                        }
#pragma unroll
                    for (int t = 0; t < kTiles; ++t) {
                        union {
                            i16x4 half[2];
                            bf16x8 all;
                        } u;
                        u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(turned + (col_at ^ 32 * t)));
                        u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(turned + (col_at ^ 32 * t) + 16 * Tile<D>::kRowBytes));
                        o[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u.all, p, o[x][t], 0, 0, 0);
                    }
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup", "local");
                __builtin_amdgcn_wave_barrier();
            }

            // join the four waves' rows
            float* sums = reinterpret_cast<float*>(lds);  // [wave][register][lane]
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
                l[x] += __shfl_xor(l[x], 16, 64);
                l[x] += __shfl_xor(l[x], 32, 64);
                if (quad == 0) {
                    stat[0][wave][16 * x + n] = m[x];
                    stat[1][wave][16 * x + n] = l[x];
                }
            }
            __syncthreads();
            float top[NQ], total[NQ];
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
                top[x] = -kInf;
                total[x] = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) top[x] = fmaxf(top[x], stat[0][w][16 * x + n]);
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float mw = stat[0][w][16 * x + n], lw = stat[1][w][16 * x + n];
                    total[x] += mw == -kInf ? lw : lw * __builtin_amdgcn_exp2f(mw - top[x]);
                }
                const float f = m[x] == -kInf ? 1.0f : __builtin_amdgcn_exp2f(m[x] - top[x]);
#pragma unroll
                for (int t = 0; t < kTiles; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sums[(wave * kRegs + (x * kTiles + t) * 4 + i) * kWave + lane] = o[x][t][i] * f;
            }
            __syncthreads();
            float* part = whole ? nullptr : a.few_part + few_part_at(a, D, part_index);
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
                if (16 * x + n >= r.rows) continue;
                uint16_t* out = a.o.p + row_at(a, r, a.o, 16 * x + n);
                const float inv = total[x] == 0.0f ? 0.0f : 1.0f / total[x];
                for (int t = wave; t < kTiles; t += kWaves) {
                    f32x4 y = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int w = 0; w < kWaves; ++w)
#pragma unroll
                        for (int i = 0; i < 4; ++i) y[i] += sums[(w * kRegs + (x * kTiles + t) * 4 + i) * kWave + lane];
                    const int d = 16 * t + 4 * quad;
                    if (!whole) {
                        *reinterpret_cast<f32x4*>(part + (16 * x + n) * D + d) = y;
                    } else if (d < a.cache.dim) {
                        const bf16x2 lo = {static_cast<__bf16>(y[0] * inv), static_cast<__bf16>(y[1] * inv)};
                        const bf16x2 hi = {static_cast<__bf16>(y[2] * inv), static_cast<__bf16>(y[3] * inv)};
                        *reinterpret_cast<u32x2_any*>(out + d) =
                            u32x2{__builtin_bit_cast(unsigned int, lo), __builtin_bit_cast(unsigned int, hi)};
                    }
                }
                if (!whole && wave == 0 && quad == 0) {
                    part[a.few_rows * D + 16 * x + n] = top[x];
                    part[a.few_rows * (D + 1) + 16 * x + n] = total[x];
                }
            }
            __syncthreads();  // the next unit writes where this one's sums were
        }
    }
}

// Joins n parts of a row, row i of the `rows` that a part holds, one wave: a lane per part for the statistics,
// then a lane per column or two.  part(p) is the p-th part's first float.
template <int D, class Part>
__device__ __forceinline__ void join_row(const PagedArgs& a, const Request& r, int rows, int row, int i, int n, Part part) {
    constexpr int kPer = (D + 63) / 64, kAtOnce = 8;
    const int lane = threadIdx.x & 63;
    float m = -kInf, total = 0.0f, acc[kPer];
#pragma unroll
    for (int e = 0; e < kPer; ++e) acc[e] = 0.0f;
    for (int p0 = 0; p0 < n; p0 += kWave) {
        const bool mine = p0 + lane < n;
        const float* stat = part(mine ? p0 + lane : 0) + rows * D + i;
        const float mp = mine ? stat[0] : -kInf, lp = mine ? stat[rows] : 0.0f;
        float top = fmaxf(m, mp);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
        const float f = mp == -kInf ? 1.0f : __builtin_amdgcn_exp2f(mp - top);
        const float old = m == -kInf ? 1.0f : __builtin_amdgcn_exp2f(m - top);
        float sum = f * lp;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d, 64);
        total = total * old + sum;
        m = top;
#pragma unroll
        for (int e = 0; e < kPer; ++e) acc[e] *= old;
        const int count = min(n - p0, kWave);
        for (int p = 0; p < count; p += kAtOnce) {  // with the loads of kAtOnce parts on their way
            float x[kAtOnce][kPer];
#pragma unroll
            for (int y = 0; y < kAtOnce; ++y) {
                const float* from = part(p0 + min(p + y, count - 1)) + i * D + min(kPer * lane, D - kPer);
#pragma unroll
                for (int e = 0; e < kPer; ++e) x[y][e] = from[e];
            }
#pragma unroll
            for (int y = 0; y < kAtOnce; ++y) {
                const float fp = __shfl(f, min(p + y, count - 1), 64);
#pragma unroll
                for (int e = 0; e < kPer; ++e) acc[e] += p + y < count ? fp * x[y][e] : 0.0f;
            }
        }
    }
    const float inv = total == 0.0f ? 0.0f : 1.0f / total;
    const int d = kPer * lane;
    uint16_t* out = a.o.p + (r.q0 + row / a.group) * a.o.row + (r.head * a.group + row % a.group) * a.o.head + d;
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (d + e < a.cache.dim) out[e] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(acc[e] * inv));
}

// Joins the pieces of the rows that more than one piece holds: a workgroup per `rows` rows of a tile.
template <int D>
__global__ __launch_bounds__(kThreads) void paged_join_kernel(const PagedArgs a, int rows) {
    __shared__ int mem[kTileOfInts];
    const int groups = kTileRows / rows;
    const int64_t n = blockIdx.x / groups / a.cache.heads;
    const TileOf at = tile_of(a, n, mem);
    if (at.b < 0) return;
    const Request r = request<false>(a, at.b, static_cast<int>(blockIdx.x / groups % a.cache.heads));
    const int tile = at.tile, tile0 = tile * kTileRows, i0 = static_cast<int>(blockIdx.x % groups) * rows;
    if (tile0 + i0 >= r.rows) return;
    const Pieces ps = pieces(a, r, tile0);
    if (ps.first == ps.last) return;
    const float* first = a.tile_part + part_at(a, D, r.head, n, ps.first);
    const int64_t piece_floats = static_cast<int64_t>(kTileRows) * (D + 2);
    for (int i = i0 + (threadIdx.x >> 6); i < i0 + rows && tile0 + i < r.rows; i += kWaves)
        join_row<D>(a, r, kTileRows, tile0 + i, i, ps.last - ps.first + 1, [&](int p) { return first + p * piece_floats; });
}

// Joins the parts of the requests whose blocks lie in more than one share: a workgroup per request and head.
template <int D>
__global__ __launch_bounds__(kThreads) void paged_few_join_kernel(const PagedArgs a) {
    __shared__ int64_t mem[kWaves][2];
    const int64_t b = blockIdx.x / a.cache.heads;
    const Request r = request<true>(a, b, static_cast<int>(blockIdx.x % a.cache.heads));
    const Blocks bl = blocks_of(a, r);
    const Stream stream = count_blocks(a, b, mem);
    const int64_t start = stream.before, share = share_of(a, stream.all);
    const int64_t w0 = start / share;
    const int count = static_cast<int>((start + bl.n - 1) / share - w0) + 1;
    if (bl.n == 0 || count == 1) return;
    for (int i = threadIdx.x >> 6; i < r.rows; i += kWaves)
        join_row<D>(a, r, a.few_rows, i, i, count, [&](int p) {
            return a.few_part + few_part_at(a, D, 2 * ((w0 + p) * a.cache.heads + r.head) + (p == 0 && start % share != 0 ? 1 : 0));
        });
}

// -------------------------------------------------------------------------------------- slots
// Every workgroup takes the sums over all requests itself (8 bytes a request, from the cache) and
// then writes the slots of its share of the tokens, so that one launch does it.  A request's new
// pages are the next ones of the free list; the token that starts a page writes its table entry.
// Bound by the launch and a chain of four reads: 256 single tokens 4.4 us, 64 prompts of 70796 tokens 5.9 us.
__global__ __launch_bounds__(kThreads) void slots_kernel(const SlotArgs a) {
    __shared__ int64_t mem[kWaves][2];
    __shared__ int64_t s_first[kThreads + 1];  // token where a request of the chunk starts
    __shared__ int64_t s_page[kThreads];       // its first new page in the free list
    __shared__ int s_cached[kThreads], s_granted[kThreads];
    __shared__ int s_refused[kWaves];
    __shared__ int64_t s_taken[kWaves];
    const int tid = threadIdx.x;
    int64_t n_free = *a.n_free;
    n_free = n_free < 0 ? 0 : n_free < a.free_cap ? n_free : a.free_cap;
    Two base = {0, 0};
    int refused = 0;
    int64_t taken = 0;
    for (int64_t b0 = 0; b0 < a.batch; b0 += kThreads) {
        const int64_t b = b0 + tid;
        int64_t cached = 0, fresh = 0, need = 0;
        bool wide = false;
        if (b < a.batch) {
            cached = max(a.cached[b], 0);
            fresh = max(a.fresh[b], 0);
            const int64_t held = (cached + a.page_size - 1) / a.page_size;
            const int64_t full = (cached + fresh + a.page_size - 1) / a.page_size;
            wide = full > a.width;
            need = wide ? 0 : full - held;
        }
        Two total;
        const Two at = scan({fresh, need}, &total, mem);
        const int64_t first = base.tokens + at.tokens, page = base.pages + at.pages;
        const bool granted = !wide && (fresh == 0 || first + fresh <= a.n_slots) && (need == 0 || page + need <= n_free);
        s_first[tid] = first;
        s_page[tid] = page;
        s_cached[tid] = static_cast<int>(cached);
        s_granted[tid] = granted ? 1 : 0;
        if (tid == 0) s_first[kThreads] = base.tokens + total.tokens;
        if (b < a.batch) {
            refused += granted ? 0 : 1;
            if (granted && need > 0) taken = page + need;
            if (blockIdx.x == 0) {
                a.q_start[b] = static_cast<int32_t>(first < a.n_slots ? first : a.n_slots);
                a.kv_len[b] = granted ? static_cast<int32_t>(cached + fresh) : 0;
            }
        }
        __syncthreads();
        const int64_t t0 = base.tokens, t1 = min(base.tokens + total.tokens, a.n_slots);
        // blocks of kThreads tokens go to the workgroups in turn
        const int64_t grid = gridDim.x;
        int64_t block = t0 / kThreads;
        block += (blockIdx.x - block % grid + grid) % grid;
        for (; block * kThreads < t1; block += grid) {
            const int64_t t = block * kThreads + tid;
            if (t < t0 || t >= t1) continue;
            int lo = 0, hi = kThreads - 1;  // the last request that starts at or before t
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if (s_first[mid] <= t) lo = mid;
                else hi = mid - 1;
            }
            int64_t slot = -1;
            if (s_granted[lo]) {
                const int64_t cached_lo = s_cached[lo], place = cached_lo + t - s_first[lo];
                const int64_t column = place / a.page_size, held = (cached_lo + a.page_size - 1) / a.page_size;
                int32_t* entry = a.table + (b0 + lo) * a.width + column;
                int64_t p;
                if (column < held) {
                    p = *entry;
                } else {
                    p = a.free_pages[s_page[lo] + column - held];
                    if (p < 0 || p >= a.n_pages) p = -1;
                    if (place % a.page_size == 0) *entry = static_cast<int32_t>(p);
                }
                if (p >= 0 && p < a.n_pages) slot = p * a.page_size + place % a.page_size;
            }
            a.slots[t] = slot;
        }
        base.tokens += total.tokens;
        base.pages += total.pages;
        __syncthreads();
    }
    for (int64_t t = base.tokens + static_cast<int64_t>(blockIdx.x) * kThreads + tid; t < a.n_slots;
         t += static_cast<int64_t>(gridDim.x) * kThreads)
        a.slots[t] = -1;
    if (blockIdx.x == 0) {
        for (int d = 32; d > 0; d /= 2) {
            refused += __shfl_xor(refused, d, 64);
            taken = max(taken, static_cast<int64_t>(__shfl_xor(taken, d, 64)));
        }
        if ((tid & 63) == 0) {
            s_refused[tid >> 6] = refused;
            s_taken[tid >> 6] = taken;
        }
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kWaves; ++w) {
                s_refused[0] += s_refused[w];
                s_taken[0] = max(s_taken[0], s_taken[w]);
            }
            a.taken[0] = static_cast<int32_t>(s_taken[0]);
            a.taken[1] = s_refused[0];
            a.q_start[a.batch] = static_cast<int32_t>(min(base.tokens, a.n_slots));
        }
    }
}

// ------------------------------------------------------------------------------------- append
// Pieces of 16 bytes, those of a token head after head, first of K, then of V.  A thread takes kPieces at a
// time, all their slots and then all their bytes on the way together.  STREAM: more bytes than the L2s
// hold (32 MB) go past them (16 x 512..2048 tokens, 8 heads of 128, 129 MB read and written: 28.1 us with
// ordinary stores, 21.0 us so, 6.1 TB/s); fewer stay for the attention that reads them next.
constexpr int kPieces = 4;
constexpr int64_t kStreamBytes = 32 << 20;

template <bool STREAM>
__global__ __launch_bounds__(kThreads) void append_kernel(const Cache c, const Heads k, const Heads v,
                                                          const int64_t* __restrict__ slots, int64_t tokens) {
    const unsigned chunks = c.dim / 8, row = c.heads * chunks, per = 2 * row;
    const int64_t most = c.n_pages * c.page_size, n = tokens * per;
    const bool small = most <= 0xFFFFFFFFll;  // 32-bit division does
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * kThreads * kPieces; base < n;
         base += static_cast<int64_t>(gridDim.x) * kThreads * kPieces) {
        const int64_t t0 = base / per;
        const unsigned first = static_cast<unsigned>(base - t0 * per);
        int64_t t[kPieces], slot[kPieces];
        unsigned y[kPieces];
        u32x4 data[kPieces];
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const unsigned x = first + threadIdx.x + kThreads * i;
            y[i] = x % per;
            t[i] = t0 + x / per;
            slot[i] = slots[min(t[i], tokens - 1)];
        }
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const unsigned z = y[i] < row ? y[i] : y[i] - row, head = z / chunks;
            const Heads& from = y[i] < row ? k : v;
            data[i] = load_global(from.p + min(t[i], tokens - 1) * from.row + head * from.head + 8 * (z - head * chunks));
        }
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            if (t[i] >= tokens || slot[i] < 0 || slot[i] >= most) continue;
            const unsigned z = y[i] < row ? y[i] : y[i] - row, head = z / chunks;
            const int64_t page = small ? static_cast<unsigned>(slot[i]) / static_cast<unsigned>(c.page_size) : slot[i] / c.page_size;
            uint16_t* to = (y[i] < row ? c.k : c.v) + page * c.page + (slot[i] - page * c.page_size) * c.row + head * c.head +
                           8 * (z - head * chunks);
            if constexpr (STREAM) __builtin_nontemporal_store(data[i], reinterpret_cast<u32x4_any*>(to));
            else *reinterpret_cast<u32x4_any*>(to) = data[i];
        }
    }
}

template <int D>
hipError_t launch_paged(const PagedArgs& a, hipStream_t stream) {
    const int64_t units = a.batch * a.cache.heads;
    hipError_t e = hipSuccess;
    if (a.tiles > 0) {
        const unsigned tiles = static_cast<unsigned>(a.tile_count * a.cache.heads), grid = tiles * a.splits;
        if (aligned_pieces({a.cache.k, a.cache.page, a.cache.row, a.cache.head}) && reinterpret_cast<uintptr_t>(a.cache.v) % 16 == 0)
            e = launch(paged_kernel<D, true>, dim3(grid), kThreads, stream, a);
        else e = launch(paged_kernel<D, false>, dim3(grid), kThreads, stream, a);
        if (e == hipSuccess && a.splits > 1) {
            const int rows = join_rows(tiles);
            static_assert(join_rows(1) % kWaves == 0 && join_rows(1 << 20) % kWaves == 0, "whole rounds of the waves");
            e = launch(paged_join_kernel<D>, dim3(tiles * (kTileRows / rows)), kThreads, stream, a, rows);
        }
    }
    if (e == hipSuccess && a.few_rows > 0) {
        const bool full = a.cache.dim == D;
        const unsigned grid = static_cast<unsigned>(a.shares > 0 ? static_cast<int64_t>(a.shares) * a.cache.heads : units);
        if (a.few_rows == 16 && full) e = launch(paged_few_kernel<D, 1, true>, dim3(grid), kThreads, stream, a);
        else if (a.few_rows == 16) e = launch(paged_few_kernel<D, 1, false>, dim3(grid), kThreads, stream, a);
        else if (full) e = launch(paged_few_kernel<D, 2, true>, dim3(grid), kThreads, stream, a);
        else e = launch(paged_few_kernel<D, 2, false>, dim3(grid), kThreads, stream, a);
        if (e == hipSuccess && a.shares > 0)
            e = launch(paged_few_join_kernel<D>, dim3(static_cast<unsigned>(units)), kThreads, stream, a);
    }
    return e;
}

}  // namespace

hipError_t launch_attention_paged(const PagedArgs& a, hipStream_t stream) {
    switch (padded_dim(a.cache.dim)) {
        case 64: return launch_paged<64>(a, stream);
        case 96: return launch_paged<96>(a, stream);
        default: return launch_paged<128>(a, stream);
    }
}

hipError_t launch_cache_slots(const SlotArgs& a, int n_cu, hipStream_t stream) {
    const int64_t blocks = (a.n_slots + kThreads - 1) / kThreads;
    const unsigned grid = static_cast<unsigned>(blocks < 1 ? 1 : blocks < n_cu ? blocks : n_cu);
    return launch(slots_kernel, dim3(grid), kThreads, stream, a);
}

hipError_t launch_cache_append(const Cache& c, const Heads& k, const Heads& v, const int64_t* slots, int64_t tokens,
                               int n_cu, hipStream_t stream) {
    if (tokens == 0 || c.heads == 0) return hipSuccess;
    const int64_t pieces = tokens * 2 * c.heads * (c.dim / 8), blocks = (pieces + kThreads * kPieces - 1) / (kThreads * kPieces);
    const int64_t most = 64 * static_cast<int64_t>(n_cu);
    const unsigned grid = static_cast<unsigned>(blocks < most ? blocks : most);
    if (16 * pieces > kStreamBytes) return launch(append_kernel<true>, dim3(grid), kThreads, stream, c, k, v, slots, tokens);
    return launch(append_kernel<false>, dim3(grid), kThreads, stream, c, k, v, slots, tokens);
}

}  // namespace bsm_att
