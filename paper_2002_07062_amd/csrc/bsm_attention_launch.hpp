// Attention launches: what the C-ABI layer hands to the kernels (internal).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <tuple>

namespace bsm_att {

// One piece of work of a plan: 128 rows (kTileRows) of one head of one sequence, query rows for the
// forward pass and dq, key rows for dk and dv.  A unit without rows (rows == 0) does nothing.
struct Unit {
    int64_t q_start, kv_start;  // the sequence's first row in the caller's tensors
    int64_t lse_row;            // its first query row in the compact numbering of the plan
    int64_t part_row;           // first row of the unit's parts (see SequenceArgs)
    int32_t seq, head;          // head: query head, or key/value head
    int32_t first, rows;        // the unit's rows within the sequence
    int32_t q_len, kv_len;
    int32_t part, parts;        // which of the unit's workgroups this is
};
static_assert(sizeof(Unit) == 64, "");

constexpr int kTileRows = 128;

// hipLaunchKernel reports a failed launch itself: the thread's last error may be another call's.
template <class... P, class... A>
hipError_t launch(void (*kernel)(P...), dim3 grid, unsigned threads, hipStream_t stream, const A&... args) {
    std::tuple<P...> values(args...);
    return std::apply(
        [&](auto&... x) {
            void* at[] = {&x...};
            return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), at, 0, stream);
        },
        values);
}

// What the kernels pad a head dimension to.
constexpr int padded_dim(int dim) { return dim <= 64 ? 64 : dim <= 96 ? 96 : 128; }

// A caller's tensor: element (b, row, head, d) at p + b seq + row row + head head + d.
struct Heads {
    uint16_t* p;
    int64_t seq, row, head;
};

// The most rows and keys of a sequence, tokens of a paged call, and keys of a request.
constexpr int32_t kMostRows = 1 << 30;

// window 0: none; of a larger one than kMostRows, which hides as little, the kernels get that: a position from -kMostRows
// on less the window then fits 32 bits.  (With p >= window compared first, any window would do, but dq of heads over 96
// spills two registers more: gradient of 4 x 4096 causal rows, 32/8 heads of 128, 2116 .. 2153 us, 2084 .. 2114 so.)
struct Mask {
    int32_t causal, window;
};
constexpr int32_t held_window(int32_t window) { return window < kMostRows ? window : kMostRows; }

struct SequenceArgs {
    Heads q, k, v, o, dout, dq, dk, dv;
    float* lse;       // [heads_q][total_q]
    float* delta;     // [heads_q][total_q]: sum of dout * o over a row (backward)
    int64_t total_q;
    int32_t group;    // query heads per key/value head
    int32_t dim;
    int32_t unit_rows;  // query rows of a query unit: kTileRows, or half of them
    int32_t key_rows;   // keys of a key unit: kTileRows, or of head dimensions up to 64 half of them
    int32_t few_units;  // these run at once, two workgroups on a CU, and have more than 64 keys
    Mask mask;
    float scale;
    // Sums of units that several workgroups share, a range of the steps each: row r of part p is row part_row +
    // p rows + r of [row][dk, dv][padded_dim] or [row][padded_dim] fp32; added up in order.
    float *part, *dq_part;
};

bool aligned_pieces(const Heads& t);  // 16-byte pieces on 16-byte boundaries

hipError_t launch_attention(const SequenceArgs& a, const Unit* units, int64_t n, hipStream_t stream);
// The units of a gradient: dq's, those of dk and dv, and the units of both that have parts.
struct GradientUnits {
    const Unit *q, *kv, *joins;  // the joins of dk and dv follow those of dq
    int64_t n_q, n_kv, n_q_joins, n_kv_joins;
};
// dq (and delta), then dk and dv, which read delta, and the joins
hipError_t launch_attention_backward(const SequenceArgs& a, const GradientUnits& u, hipStream_t stream);

// ------------------------------------------------------------------------------ paged cache
struct Cache {
    uint16_t *k, *v;
    int64_t page, row, head;  // strides in elements
    int64_t n_pages;
    int32_t page_size, heads, dim;
};

struct PagedArgs {
    Cache cache;
    Heads q, o;               // seq strides are not used: rows are token indices
    const int32_t* table;     // [batch][width]
    const int32_t* q_start;   // [batch + 1]
    const int32_t* kv_len;    // [batch]
    int64_t batch, tokens;
    int32_t width, max_q;
    int32_t group;
    int32_t window;
    float scale;
    // how the work is cut, from bounds on the lengths alone
    // Requests of up to few_rows rows of a key/value head (16 or 32; 0: none) go by shares: equal shares of
    // their blocks of kFewKeys keys (see share_of), of which `round` for each head give every CU one; shares 0: one
    // request each.
    int32_t few_rows, shares, round;
    // The others go by tiles of kTileRows rows, `tiles` per request and key/value head (0: there are none),
    // in `splits` pieces of the key axis of split_keys keys each, a multiple of kKeyTile.
    int32_t tiles, splits, split_keys;
    int64_t tile_count;  // tiles with rows, of one head, at most
    float *few_part, *tile_part;  // outputs and statistics of what has to be joined
};

constexpr int kKeyTile = 128;
// Rows of a tile that a workgroup joins, where `tiles` of all heads have pieces to join: a wave takes four of them one
// after the other, but one where that leaves few workgroups (a chunk of 16 tokens over 16384 keys, 32/8 heads of 128:
// 52 us with four, 30 us with one).
constexpr int join_rows(int64_t tiles) { return tiles < 128 ? 4 : 16; }
constexpr int kFewKeys = 128, kFewestBlocks = 4, kMostBlocks = 16;  // of a share, see share_of

hipError_t launch_attention_paged(const PagedArgs& a, hipStream_t stream);

struct SlotArgs {
    const int32_t *cached, *fresh;
    int64_t batch;
    int32_t page_size, width;
    int64_t n_pages;
    int32_t* table;           // [batch][width]
    const int32_t* free_pages;
    int64_t free_cap;         // entries of free_pages
    const int32_t* n_free;
    int32_t *q_start, *kv_len;
    int64_t* slots;
    int64_t n_slots;
    int32_t* taken;           // [2]
};

hipError_t launch_cache_slots(const SlotArgs& a, int n_cu, hipStream_t stream);

hipError_t launch_cache_append(const Cache& c, const Heads& k, const Heads& v, const int64_t* slots, int64_t tokens,
                               int n_cu, hipStream_t stream);

}  // namespace bsm_att
