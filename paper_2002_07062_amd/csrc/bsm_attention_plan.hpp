// Host planner of attention over ragged sequences: sequence lengths -> work units in the order of
// the schedule.  Pure C++17, no HIP runtime calls.
#pragma once

#include <cstdint>
#include <vector>

#include "bsm.h"
#include "bsm_attention_launch.hpp"

namespace bsm_att {

struct Sequences {
    int64_t batch = 0;
    std::vector<int32_t> q_len, kv_len;
    std::vector<int64_t> q_start, kv_start;  // first rows in the operands
    int32_t heads_q = 1, heads_kv = 1, dim = 8;
    Mask mask{0, 0};
    int64_t total_q = 0, total_kv = 0;
    int64_t q_end = 0, kv_end = 0;           // largest row + 1
    int64_t q_longest = 0, kv_longest = 0;   // rows of the longest sequence
    bool q_in_order = true, kv_in_order = true;  // no sequence starts before the one before it
    bool q_shared = false, kv_shared = false;  // some row belongs to two sequences
    int64_t pairs = 0;
};

// Fills the starts (packed where null) and the totals from the lengths.
void finish_sequences(Sequences* s, const int64_t* q_start, const int64_t* kv_start);

// Rows of the forward pass's query units: 128, or 64 where the longest of 128 would outlast the others.
int32_t query_rows(const Sequences& s, int n_cu);
// Keys of the units of dk and dv: 128, or 64 where there is little to do.
int32_t key_rows(const Sequences& s, int n_cu);

// Units of `rows` query rows (forward pass, dq), or of keys (dk, dv), in launch order; the unit of
// workgroup w is expected to run on XCD w mod n_xcd.  Where `slots` workgroups run at once, units that
// would outlast the others are cut into parts (with_care: only by much); slots 0: none is.
struct Units {
    std::vector<Unit> units, joins;  // joins: the units with parts
    int64_t part_rows = 0;           // rows of all parts
};
Units make_units(const Sequences& s, bool of_keys, int32_t rows, int64_t slots, bool with_care, bsm_schedule schedule, int n_xcd);

// How attention over a paged cache is cut.
struct PagedCut {
    int32_t few_rows, shares, round, tiles, splits, split_keys;  // as in PagedArgs
    int64_t tile_count;
    int64_t few_floats, tile_floats;                                   // of the parts
    int64_t grid;                                                      // workgroups of the largest launch
};
PagedCut cut_paged(int64_t batch, int64_t tokens, int32_t heads_kv, int32_t group, int32_t dim, int32_t max_q,
                   int32_t max_kv, int n_cu);

}  // namespace bsm_att
