// The paged key/value cache: attention of new tokens over the pages, the slots of new tokens, and
// the copy of their keys and values into the slots.
#include "bsm_attention.hpp"

namespace bsm_att {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = 4;

// ---------------------------------------------------------------------------------- attention
// One request and key/value head: the rows are (new token, query head of the group) pairs, token
// after token, so that the query heads that share a key/value head read it once.
struct Request {
    int b, head;       // request, key/value head
    int64_t q0;        // its first row in q and o
    int q_len, kv_len;
    int rows;          // q_len (at most max_q) * group
};

__device__ __forceinline__ Request request(const PagedArgs& a, int64_t unit) {
    Request r;
    r.b = static_cast<int>(unit / a.cache.heads);
    r.head = static_cast<int>(unit % a.cache.heads);
    const int64_t q0 = a.q_start[r.b], q1 = a.q_start[r.b + 1];
    r.q0 = q0 < 0 ? 0 : q0 < a.tokens ? q0 : a.tokens;
    const int64_t e = q1 < r.q0 ? r.q0 : q1 < a.tokens ? q1 : a.tokens;
    r.q_len = static_cast<int>(e - r.q0);
    const int64_t most = static_cast<int64_t>(a.width) * a.cache.page_size;
    const int kv = a.kv_len[r.b];
    r.kv_len = kv < 0 ? 0 : kv < most ? kv : static_cast<int>(most);
    r.rows = min(r.q_len, a.max_q) * a.group;
    return r;
}

struct Keys {
    int lo, hi;  // seen keys
};
__device__ __forceinline__ Keys seen_keys(const PagedArgs& a, const Request& r, int token) {
    const int p = token + r.kv_len - r.q_len;
    Keys k = {0, p < r.kv_len - 1 ? p : r.kv_len - 1};
    if (a.window > 0 && p - a.window + 1 > 0) k.lo = p - a.window + 1;
    return k;
}

// Pieces of the key axis that a tile of rows needs: first .. last, each split_keys keys from
// piece * split_keys (the last one of the grid: all that is left).
struct Pieces {
    Keys keys;  // seen by some row of the tile
    int first, last;
};
__device__ __forceinline__ Pieces pieces(const PagedArgs& a, const Request& r, int r0) {
    const int r1 = min(r0 + a.tile_rows, r.rows) - 1;
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

// Floats of one piece's part: its rows' outputs, then their references and sums.
__device__ __forceinline__ int64_t part_at(const PagedArgs& a, int D, int64_t unit, int tile, int piece) {
    return ((unit * a.tiles + tile) * a.splits + piece) * a.tile_rows * (D + 2);
}

// The rows of K and V that a thread stages: tile row i is key j0 + i of the request.  Keys past its
// end, and keys of table entries that name no page, are zeros.
template <int D, int ROWS, int THREADS>
struct PagedStage {
    using S = Stage<D, ROWS, THREADS>;
    S k, v;
    int page[S::kN];
    __device__ __forceinline__ static int divide(const PagedArgs& a, int j) { return j / a.cache.page_size; }
    // table entries of the tile at j0 (-1: none)
    __device__ __forceinline__ void find(const PagedArgs& a, const int32_t* table, int tid, int j0, int end) {
#pragma unroll
        for (int n = 0; n < S::kN; ++n) {
            const int j = j0 + S::row(tid, n);
            page[n] = j < end ? table[divide(a, j)] : -1;
        }
    }
    __device__ __forceinline__ void load(const PagedArgs& a, int head, int tid, int j0, int chunks) {
        const int c = S::chunk(tid);
#pragma unroll
        for (int n = 0; n < S::kN; ++n) {
            const int j = j0 + S::row(tid, n);
            k.r[n] = v.r[n] = u32x4{0, 0, 0, 0};
            if (page[n] >= 0 && page[n] < a.cache.n_pages && c < chunks) {
                const int64_t at = page[n] * a.cache.page + (j - divide(a, j) * a.cache.page_size) * a.cache.row +
                                   head * a.cache.head + 8 * c;
                k.r[n] = *reinterpret_cast<const u32x4_any*>(a.cache.k + at);
                v.r[n] = *reinterpret_cast<const u32x4_any*>(a.cache.v + at);
            }
        }
    }
};

template <int D>
__device__ __forceinline__ void put_part(float* part, int tile_rows, int row, const f32x16& acc, int t, int h) {
#pragma unroll
    for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(part + static_cast<int64_t>(row) * D + 32 * t + 8 * g + 4 * h) =
            f32x4{acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]};
    (void)tile_rows;
}

// TEAM 4: a tile has 128 rows, 32 per wave, and the waves share the staged keys.
// TEAM 1: a tile has 32 rows, the waves take turns at blocks of 32 keys, each staging its own, and
// join their rows at the end: few rows over many keys (decode) are bound by reading the cache, and
// four waves that never wait for each other keep more of it in flight.
template <int D, int TEAM>
__global__ __launch_bounds__(kThreads, 2) void paged_kernel(const PagedArgs a) {
    constexpr int kKeys = TEAM == 4 ? 64 : 32;
    constexpr int kTeamThreads = TEAM * kWave;
    constexpr int kBuffers = TEAM == 4 ? 2 : 1;
    constexpr int kTileElems = kKeys * D;
    __shared__ __align__(16) uint16_t lds[kBuffers * (4 / TEAM) * 2 * kTileElems];
    __shared__ float stat[2][4][kRows];
    const int64_t units = a.batch * a.cache.heads;
    const int64_t unit = blockIdx.x % units;
    const int rest = static_cast<int>(blockIdx.x / units);
    const int tile = rest % a.tiles, piece = rest / a.tiles;
    const Request r = request(a, unit);
    const int tile0 = tile * a.tile_rows;
    if (tile0 >= r.rows) return;
    const Pieces ps = pieces(a, r, tile0);
    if (piece < ps.first || piece > ps.last) return;

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, li = lane & 31, h = lane >> 5;
    const int chunks = a.cache.dim / 8;
    const int row0 = TEAM == 4 ? tile0 + kRows * wave : tile0;  // of the wave
    const int row = row0 + li;
    const bool live = row < r.rows;
    const bool any_row = row0 < r.rows;
    const int token = row / a.group, q_head = r.head * a.group + row % a.group;
    const int64_t q_row = r.q0 + token;
    RowOperand<D> q;
    q.load(a.q.p + q_row * a.q.row + q_head * a.q.head, live, h, chunks);
    const Keys mine = seen_keys(a, r, token);
    const Keys w0 = seen_keys(a, r, row0 / a.group), w1 = seen_keys(a, r, (row0 + kRows - 1) / a.group);

    const int team_tid = TEAM == 4 ? tid : lane;
    const int step = TEAM == 4 ? kKeys : kKeys * kWaves;
    const int from = max(ps.keys.lo, piece * a.split_keys);
    const int end = piece == a.splits - 1 ? ps.keys.hi + 1 : min(ps.keys.hi + 1, (piece + 1) * a.split_keys);
    const int begin = from / kKeys * kKeys + (TEAM == 4 ? 0 : wave * kKeys);
    const int32_t* table = a.table + static_cast<int64_t>(r.b) * a.width;
    uint16_t* mem = lds + (TEAM == 4 ? 0 : wave * 2 * kTileElems);

    Online<D> st;
    st.init();
    const float c = a.scale * kLog2e;
    PagedStage<D, kKeys, kTeamThreads> stage;
    if (begin < end) {
        stage.find(a, table, team_tid, begin, r.kv_len);
        stage.load(a, r.head, team_tid, begin, chunks);
        stage.find(a, table, team_tid, begin + step, r.kv_len);
        if (TEAM == 4) {
            stage.k.store(team_tid, mem);
            stage.v.store(team_tid, mem + kTileElems);
        }
    }
    int buf = 0;
    for (int j0 = begin; j0 < end; j0 += step) {
        const int next = j0 + step;
        if (TEAM == 4) {
            lds_barrier();
        } else {
            stage.k.store(team_tid, mem);
            stage.v.store(team_tid, mem + kTileElems);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup", "local");
            __builtin_amdgcn_wave_barrier();
        }
        if (next < end) {
            stage.load(a, r.head, team_tid, next, chunks);
            stage.find(a, table, team_tid, next + step, r.kv_len);
        }
        const uint16_t* now = mem + buf * 2 * kTileElems;
        if (any_row && j0 <= w1.hi && j0 + kKeys > w0.lo) {
            f32x16 s[kKeys / 32];
#pragma unroll
            for (int k = 0; k < kKeys / 32; ++k) s[k] = row_product<D>(now, 32 * k, q, lane);
            if (j0 < w1.lo || j0 + kKeys - 1 > w0.hi || end < j0 + kKeys) {
#pragma unroll
                for (int k = 0; k < kKeys / 32; ++k) mask_block(s[k], j0 + 32 * k, h, mine.lo, min(mine.hi, end - 1));
            }
            st.weigh(s, c);
#pragma unroll
            for (int k = 0; k < kKeys / 32; ++k) col_product<D>(st.o, now + kTileElems, 32 * k, s[k], lane);
        }
        if (TEAM == 4) {
            if (next < end) {
                buf ^= 1;
                stage.k.store(team_tid, mem + buf * 2 * kTileElems);
                stage.v.store(team_tid, mem + buf * 2 * kTileElems + kTileElems);
            }
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup", "local");
            __builtin_amdgcn_wave_barrier();
        }
    }

    const bool whole = ps.first == ps.last;
    float* part = whole ? nullptr : a.part + part_at(a, D, unit, tile, piece);
    uint16_t* out = a.o.p + q_row * a.o.row + q_head * a.o.head;
    float total = st.row_sum();
    if (TEAM == 4) {
        if (whole) {
            store_row<D>(out, live, st.o, total == 0.0f ? 0.0f : 1.0f / total, h, chunks);
        } else if (live) {
#pragma unroll
            for (int t = 0; t < D / 32; ++t) put_part<D>(part, a.tile_rows, row - tile0, st.o[t], t, h);
            if (h == 0) {
                part[a.tile_rows * D + row - tile0] = st.m;
                part[a.tile_rows * (D + 1) + row - tile0] = total;
            }
        }
        return;
    }
    // join the four waves' rows
    float* sums = reinterpret_cast<float*>(lds);  // [wave][register][lane]
    constexpr int kRegs = D / 2;
    static_assert(sizeof(lds) >= 4 * kRegs * kWave * sizeof(float) || TEAM == 4, "");
    if (h == 0) {
        stat[0][wave][li] = st.m;
        stat[1][wave][li] = total;
    }
    __syncthreads();
    float m = -kInf;
#pragma unroll
    for (int w = 0; w < 4; ++w) m = fmaxf(m, stat[0][w][li]);
    total = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w)
        total += stat[0][w][li] == -kInf ? stat[1][w][li] : stat[1][w][li] * __builtin_amdgcn_exp2f(stat[0][w][li] - m);
    const float f = st.m == -kInf ? 1.0f : __builtin_amdgcn_exp2f(st.m - m);
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[(wave * kRegs + 16 * t + i) * kWave + lane] = st.o[t][i] * f;
    __syncthreads();
    if (wave >= D / 32) return;
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float x = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) x += sums[(w * kRegs + 16 * wave + i) * kWave + lane];
        acc[i] = x;
    }
    if (whole) {
        store_block(out, live, acc, total == 0.0f ? 0.0f : 1.0f / total, wave, h, chunks);
    } else if (live) {
        put_part<D>(part, a.tile_rows, row - tile0, acc, wave, h);
        if (h == 0 && wave == 0) {
            part[a.tile_rows * D + row - tile0] = m;
            part[a.tile_rows * (D + 1) + row - tile0] = total;
        }
    }
}

// Joins the pieces of the rows that more than one piece holds: one wave per row.
template <int D>
__global__ __launch_bounds__(kThreads) void paged_join_kernel(const PagedArgs a) {
    const int64_t units = a.batch * a.cache.heads;
    const int64_t unit = blockIdx.x % units;
    const int tile = static_cast<int>(blockIdx.x / units);
    const Request r = request(a, unit);
    const int tile0 = tile * a.tile_rows;
    if (tile0 >= r.rows) return;
    const Pieces ps = pieces(a, r, tile0);
    if (ps.first == ps.last) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int kPer = D / 64;
    const int64_t piece_floats = static_cast<int64_t>(a.tile_rows) * (D + 2);
    for (int i = wave; i < a.tile_rows && tile0 + i < r.rows; i += kWaves) {
        const float* part = a.part + part_at(a, D, unit, tile, ps.first);
        const float* m_at = part + a.tile_rows * D + i;
        const float* l_at = m_at + a.tile_rows;
        float m = -kInf;
        for (int p = 0; p <= ps.last - ps.first; ++p) m = fmaxf(m, m_at[p * piece_floats]);
        float total = 0.0f, acc[kPer];
#pragma unroll
        for (int e = 0; e < kPer; ++e) acc[e] = 0.0f;
        for (int p = 0; p <= ps.last - ps.first; ++p) {
            const float mp = m_at[p * piece_floats];
            const float f = mp == -kInf ? 1.0f : __builtin_amdgcn_exp2f(mp - m);
            total += f * l_at[p * piece_floats];
#pragma unroll
            for (int e = 0; e < kPer; ++e) acc[e] += f * part[p * piece_floats + static_cast<int64_t>(i) * D + kPer * lane + e];
        }
        const float inv = total == 0.0f ? 0.0f : 1.0f / total;
        const int row = tile0 + i, d = kPer * lane;
        uint16_t* out = a.o.p + (r.q0 + row / a.group) * a.o.row + (r.head * a.group + row % a.group) * a.o.head + d;
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (d + e < a.cache.dim) out[e] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(acc[e] * inv));
    }
}

// -------------------------------------------------------------------------------------- slots
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

// Every workgroup takes the sums over all requests itself (8 bytes a request, from the cache) and
// then writes the slots of its share of the tokens, so that one launch does it.  A request's new
// pages are the next ones of the free list; the token that starts a page writes its table entry.
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
        const bool granted = !wide && first + fresh <= a.n_slots && (need == 0 || page + need <= n_free);
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
// Piece x of 16 bytes of a token: its chunks head after head, first those of K, then those of V.
__global__ __launch_bounds__(kThreads) void append_kernel(const Cache c, const Heads k, const Heads v,
                                                          const int64_t* __restrict__ slots, int64_t tokens) {
    const int chunks = c.dim / 8, row = c.heads * chunks, per = 2 * row;
    const int64_t n = tokens * per, step = static_cast<int64_t>(gridDim.x) * kThreads;
    for (int64_t x = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; x < n; x += step) {
        const int64_t t = x / per;
        int y = static_cast<int>(x - t * per);
        const int64_t slot = slots[t];
        if (slot < 0 || slot >= c.n_pages * c.page_size) continue;
        const bool is_v = y >= row;
        y -= is_v ? row : 0;
        const int head = y / chunks, e = 8 * (y - head * chunks);
        const Heads& from = is_v ? v : k;
        const int64_t page = slot / c.page_size;
        uint16_t* to = (is_v ? c.v : c.k) + page * c.page + (slot - page * c.page_size) * c.row + head * c.head + e;
        *reinterpret_cast<u32x4_any*>(to) = *reinterpret_cast<const u32x4_any*>(from.p + t * from.row + head * from.head + e);
    }
}

template <int D>
hipError_t launch_paged(const PagedArgs& a, hipStream_t stream) {
    const int64_t tiles = a.batch * a.cache.heads * a.tiles;
    const unsigned grid = static_cast<unsigned>(tiles * a.splits);
    if (a.tile_rows == kRows) paged_kernel<D, 1><<<grid, kThreads, 0, stream>>>(a);
    else paged_kernel<D, 4><<<grid, kThreads, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    paged_join_kernel<D><<<static_cast<unsigned>(tiles), kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_paged(const PagedArgs& a, hipStream_t stream) {
    return a.cache.dim <= 64 ? launch_paged<64>(a, stream) : launch_paged<128>(a, stream);
}

hipError_t launch_cache_slots(const SlotArgs& a, int n_cu, hipStream_t stream) {
    const int64_t blocks = (a.n_slots + kThreads - 1) / kThreads;
    const unsigned grid = static_cast<unsigned>(blocks < 1 ? 1 : blocks < n_cu ? blocks : n_cu);
    slots_kernel<<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_cache_append(const Cache& c, const Heads& k, const Heads& v, const int64_t* slots, int64_t tokens,
                               int n_cu, hipStream_t stream) {
    if (tokens == 0 || c.heads == 0) return hipSuccess;
    const int64_t pieces = tokens * 2 * c.heads * (c.dim / 8), blocks = (pieces + kThreads - 1) / kThreads;
    const int64_t most = 8 * static_cast<int64_t>(n_cu);
    append_kernel<<<static_cast<unsigned>(blocks < most ? blocks : most), kThreads, 0, stream>>>(c, k, v, slots, tokens);
    return hipGetLastError();
}

}  // namespace bsm_att
