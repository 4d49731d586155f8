#include "bsm_attention_plan.hpp"

#include <algorithm>
#include <functional>
#include <limits>
#include <numeric>

namespace bsm_att {
namespace {

constexpr int kStep = 64;  // keys or query rows that a workgroup takes at a time

bool any_shared(const std::vector<int64_t>& start, const std::vector<int32_t>& len) {
    std::vector<std::pair<int64_t, int64_t>> spans;
    for (size_t b = 0; b < start.size(); ++b)
        if (len[b] > 0) spans.emplace_back(start[b], start[b] + len[b]);
    std::sort(spans.begin(), spans.end());
    for (size_t i = 1; i < spans.size(); ++i)
        if (spans[i].first < spans[i - 1].second) return true;
    return false;
}

int64_t fill(const int64_t* given, const std::vector<int32_t>& len, std::vector<int64_t>* start, int64_t* end, int64_t* longest,
             bool* shared, bool* in_order) {
    int64_t total = 0;
    *end = *longest = 0;
    *in_order = true;
    start->resize(len.size());
    for (size_t b = 0; b < len.size(); ++b) {
        (*start)[b] = given ? given[b] : total;
        total += len[b];
        if (len[b] > 0) *end = std::max(*end, (*start)[b] + len[b]);
        *longest = std::max<int64_t>(*longest, len[b]);
        if (b > 0 && (*start)[b] < (*start)[b - 1]) *in_order = false;
    }
    *shared = given && any_shared(*start, len);
    return total;
}

int64_t up_to(int64_t n) { return n * (n + 1) / 2; }  // 1 + .. + n

// Pairs that the mask leaves: row i of n sees min(p + 1, window) keys, p = i + m - n, none if p < 0.
int64_t visible(int64_t n, int64_t m, Mask mask) {
    if (!mask.causal) return n * m;
    const int64_t lo = std::max<int64_t>(0, m - n), hi = m;  // rows see lo + 1 .. hi keys (those that see some)
    const int64_t w = mask.window > 0 ? mask.window : hi;
    if (w >= hi) return up_to(hi) - up_to(lo);
    if (w <= lo) return (hi - lo) * w;
    return up_to(w) - up_to(lo) + (hi - w) * w;
}

// Steps of the other axis that a unit of rows first .. first + rows - 1 takes.
int64_t query_steps(const Sequences& s, int64_t b, int64_t first, int64_t rows) {
    int64_t lo = 0, hi = s.kv_len[b];
    if (s.mask.causal) {
        const int64_t off = static_cast<int64_t>(s.kv_len[b]) - s.q_len[b];
        hi = std::min<int64_t>(hi, first + rows + off);
        if (s.mask.window > 0) lo = std::max<int64_t>(0, first + off - s.mask.window + 1);
    }
    return hi > lo ? (hi - lo / kStep * kStep + kStep - 1) / kStep : 0;
}
int64_t key_steps(const Sequences& s, int64_t b, int64_t first, int64_t rows) {
    int64_t lo = 0, hi = s.q_len[b];
    if (s.mask.causal) {
        const int64_t off = static_cast<int64_t>(s.kv_len[b]) - s.q_len[b];
        lo = std::max<int64_t>(0, first - off);
        if (s.mask.window > 0) hi = std::min<int64_t>(hi, first + rows - 1 + s.mask.window - off);
    }
    return hi > lo ? (hi - lo / kStep * kStep + kStep - 1) / kStep * (s.heads_q / s.heads_kv) : 0;
}

// Workgroups that a unit of `steps` is cut for, none of which is to take many more than `share`.  Parts of fewer
// than four steps would mostly load their rows and store their sums.
int64_t parts_of(int64_t steps, int64_t share) {
    return std::max<int64_t>(1, std::min<int64_t>({(steps + share - 1) / share, steps / 4, 64}));
}

// The share for which `slots` workgroups at a time, the longest first, are done soonest; `steps` of the units of one
// head of `heads`.  A cut costs its parts' loads and stores, two steps each, and the joining launch, four.  At best
// the slots' shares are equal; shares of up to half again as many steps can be faster, as with equal ones a few
// parts may be left over for a round of their own.  with_care: a cut has to promise 3/8 of the time.  (dq shares its CUs
// in pairs, of which one left alone runs faster: with a third less promised, the gradient of 2048 causal rows, 32/8
// heads of 128, took 212 us instead of 201; dk and dv gain from less: 1024 causal rows, 8 heads of 64, 36 us instead of
// 49.)  (The share is tried out; of many units, where it would take the host
// long, a few left over are little, and an eighth more than equal will do.)
int64_t best_share(const std::vector<int64_t>& steps, int64_t heads, int64_t slots, bool with_care) {
    int64_t total = 0, longest = 0;
    for (int64_t n : steps) {
        total += n * heads;
        longest = std::max(longest, n);
    }
    const int64_t uncut = std::max<int64_t>(1, longest), even = std::max<int64_t>(1, (total + slots - 1) / slots);
    if (even >= uncut) return uncut;
    if (static_cast<int64_t>(steps.size()) * heads > 16 * slots) return std::min(uncut, even + even / 8);
    int64_t best = 0, best_share = uncut;
    std::vector<int64_t> costs, load;
    for (int64_t share : {uncut, even, even + even / 8, even + even / 4, even + even / 2}) {
        costs.clear();
        for (int64_t n : steps)
            for (int64_t i = 0, parts = parts_of(n, share); i < parts * heads; ++i) costs.push_back(2 + (n + parts - 1) / parts);
        std::sort(costs.begin(), costs.end(), std::greater<int64_t>());
        load.assign(slots, 0);  // a heap, the least loaded slot first
        int64_t end = 0;
        for (int64_t c : costs) {
            std::pop_heap(load.begin(), load.end(), std::greater<int64_t>());
            end = std::max(end, load.back() += c);
            std::push_heap(load.begin(), load.end(), std::greater<int64_t>());
        }
        if (costs.size() > steps.size() * heads) end += 4;
        if (with_care && share != uncut) end = (8 * end + 4) / 5;
        if (best == 0 || end < best) {
            best = end;
            best_share = share;
        }
    }
    return best_share;
}

struct Costed {
    Unit unit;
    int64_t cost, kv_head;  // kv_head: index of the (sequence, key/value head) whose rows it reads
};

std::vector<Unit> order(std::vector<Costed>& units, bsm_schedule schedule, int n_xcd, int64_t kv_heads) {
    std::vector<Unit> out;
    if (schedule == BSM_SCHED_RR) {
        out.reserve(units.size());
        for (const Costed& c : units) out.push_back(c.unit);
        return out;
    }
    // The costliest key/value head goes to the least loaded XCD, and so on: the units that read the same keys
    // run on one XCD, at about the same time, and find them in its L2.
    std::vector<int64_t> cost(kv_heads, 0), by_cost(kv_heads), home(kv_heads), load(n_xcd, 0);
    for (const Costed& c : units) cost[c.kv_head] += c.cost;
    std::iota(by_cost.begin(), by_cost.end(), 0);
    std::stable_sort(by_cost.begin(), by_cost.end(), [&](int64_t x, int64_t y) { return cost[x] > cost[y]; });
    for (int64_t k : by_cost) {
        home[k] = std::min_element(load.begin(), load.end()) - load.begin();
        load[home[k]] += cost[k];
    }
    std::vector<std::vector<int64_t>> lists(n_xcd);  // longest units first
    for (size_t i = 0; i < units.size(); ++i) lists[home[units[i].kv_head]].push_back(static_cast<int64_t>(i));
    size_t longest = 0;
    for (auto& list : lists) {
        std::stable_sort(list.begin(), list.end(), [&](int64_t x, int64_t y) { return units[x].cost > units[y].cost; });
        longest = std::max(longest, list.size());
    }
    std::vector<size_t> at(n_xcd, 0);
    const Unit none{};
    if (schedule == BSM_SCHED_XCD) {
        out.reserve(longest * n_xcd);
        for (size_t i = 0; i < longest; ++i)
            for (int x = 0; x < n_xcd; ++x) out.push_back(i < lists[x].size() ? units[lists[x][i]].unit : none);
        while (!out.empty() && out.back().rows == 0) out.pop_back();
        return out;
    }
    // BALANCED: an XCD whose list is done takes from the one that has most left
    out.reserve(units.size());
    for (size_t i = 0; i < units.size(); ++i) {
        size_t x = i % n_xcd;
        if (at[x] == lists[x].size())
            for (size_t y = 0; y < lists.size(); ++y)
                if (lists[y].size() - at[y] > lists[x].size() - at[x]) x = y;
        out.push_back(units[lists[x][at[x]++]].unit);
    }
    return out;
}

}  // namespace

void finish_sequences(Sequences* s, const int64_t* q_start, const int64_t* kv_start) {
    s->total_q = fill(q_start, s->q_len, &s->q_start, &s->q_end, &s->q_longest, &s->q_shared, &s->q_in_order);
    s->total_kv = fill(kv_start, s->kv_len, &s->kv_start, &s->kv_end, &s->kv_longest, &s->kv_shared, &s->kv_in_order);
    s->pairs = 0;
    for (int64_t b = 0; b < s->batch; ++b) s->pairs += visible(s->q_len[b], s->kv_len[b], s->mask);
}

int32_t query_rows(const Sequences& s, int n_cu) {
    // A workgroup of 64 rows takes half the time of one of 128, but brings the keys in for half the rows.  It
    // pays where the longest unit takes 7/4 times an even share of what the CUs (two workgroups each) have to
    // do, for longer heads 3 times.  us, 128 and 64 rows: heads of 64, 1.9 times 63.2, 53.5 (4096 rows, 16 heads,
    // causal), an even share 88.6, 106 (the same without a mask); of 128, 3.9 times 78.6, 62.2 (8 heads, causal),
    // 2.6 times 90.3, 90.9 (12 heads, causal), twice 83.2, 86.1 (8 heads without a mask).
    int64_t total = 0, longest = 0;
    for (int64_t b = 0; b < s.batch; ++b)
        for (int64_t first = 0; first < s.q_len[b]; first += kTileRows) {
            const int64_t n = query_steps(s, b, first, std::min<int64_t>(kTileRows, s.q_len[b] - first));
            total += n * s.heads_q;
            longest = std::max(longest, n);
        }
    const int64_t quarters = padded_dim(s.dim) > 64 ? 12 : 7;
    return 4 * longest * 2 * n_cu > quarters * total ? kTileRows / 2 : kTileRows;
}

int32_t key_rows(const Sequences& s, int n_cu) {
    // A workgroup of 64 keys takes a step in about half the time of one of 128 where it is alone on its CU, but two of
    // them bring the query rows in twice.  It pays up to about four steps for each of two workgroups on a CU.  us, gradient
    // with 128 and 64 keys, heads of 64: 1.5 steps 29.4, 23.3 (2 x 512 causal rows, 12 heads), 2.3 33.6, 31.8 (3 x 600, 8/2
    // heads), 4 45.8, 45.3 (2000 rows, 4/1 heads), 16 114, 125 (4096 causal rows, 8 heads).
    if (padded_dim(s.dim) > 64) return kTileRows;
    int64_t total = 0;
    for (int64_t b = 0; b < s.batch; ++b)
        for (int64_t first = 0; first < s.kv_len[b]; first += kTileRows)
            total += key_steps(s, b, first, std::min<int64_t>(kTileRows, s.kv_len[b] - first)) * s.heads_kv;
    return total <= 4 * 2 * static_cast<int64_t>(n_cu) ? kTileRows / 2 : kTileRows;
}

Units make_units(const Sequences& s, bool of_keys, int32_t rows, int64_t slots, bool with_care, bsm_schedule schedule, int n_xcd) {
    const std::vector<int32_t>& len = of_keys ? s.kv_len : s.q_len;
    const int heads = of_keys ? s.heads_kv : s.heads_q, group = heads / s.heads_kv;
    std::vector<int64_t> steps;  // of the units of one head
    for (int64_t b = 0; b < s.batch; ++b)
        for (int64_t first = 0; first < len[b]; first += rows) {
            const int64_t n = std::min<int64_t>(rows, len[b] - first);
            steps.push_back(of_keys ? key_steps(s, b, first, n) : query_steps(s, b, first, n));
        }
    const int64_t share = slots > 0 ? best_share(steps, heads, slots, with_care) : std::numeric_limits<int32_t>::max();

    Units out;
    std::vector<Costed> units;
    int64_t lse_row = 0;
    size_t of_head = 0;
    for (int64_t b = 0; b < s.batch; ++b) {
        const size_t count = (len[b] + int64_t{rows} - 1) / rows;
        for (int head = 0; head < heads; ++head)
            for (size_t i = 0; i < count; ++i) {
                const int64_t first = static_cast<int64_t>(i) * rows, n = std::min<int64_t>(rows, len[b] - first);
                const int64_t mine = steps[of_head + i], parts = slots > 0 ? parts_of(mine, share) : 1;
                Unit u{s.q_start[b], s.kv_start[b], lse_row, out.part_rows, static_cast<int32_t>(b), head,
                       static_cast<int32_t>(first), static_cast<int32_t>(n), s.q_len[b], s.kv_len[b], 0, static_cast<int32_t>(parts)};
                if (parts > 1) {
                    out.joins.push_back(u);
                    out.part_rows += parts * n;
                }
                for (u.part = 0; u.part < u.parts; ++u.part)
                    units.push_back({u, 2 + mine / parts, b * s.heads_kv + head / group});
            }
        of_head += count;
        lse_row += s.q_len[b];
    }
    out.units = order(units, schedule, n_xcd, s.batch * s.heads_kv);
    return out;
}

PagedCut cut_paged(int64_t batch, int64_t tokens, int32_t heads_kv, int32_t group, int32_t dim, int32_t max_q,
                   int32_t max_kv, int n_cu) {
    PagedCut c{};
    const int64_t rows = std::min<int64_t>(max_q, tokens) * group, keys = std::max<int64_t>(1, max_kv);
    const int padded = padded_dim(dim);
    // Few rows over many keys are bound by reading the cache, many rows by the products: each has a kernel.  A
    // batch that may hold both launches both (one chunk of 512 tokens over 4096 and 63 single tokens over
    // 5000, 8 kv heads: 732 us by tiles alone, 377 us by both); where no request is shorter than the
    // longest chunk, or there is only one, the tiles do.
    if (rows <= 32) c.few_rows = rows <= 16 ? 16 : 32;
    else if (batch > 1 && group <= 32 && tokens < batch * max_q) c.few_rows = group <= 16 ? 16 : 32;
    if (c.few_rows > 0) {
        c.grid = batch * heads_kv;
        // A workgroup reads about 36 GB/s, the same with twice the waves.  For 9 rounds of its 128 keys, of shorter heads
        // 12, the counting of the stream and a second kernel, which joins parts, cost as much as they save (us, 8 kv
        // heads of 128, shared and not: one request of 1100 keys 18.1, 20.2, 64 of them 90.6, 61.0; heads of 64: 4 requests
        // of 1100, 2 kv heads 18.4, 13.3, 64 of up to 1500, 8 kv heads 28.8, 22.7).
        if (keys > (padded > 64 ? 1152 : 1536)) {
            // At least as many shares as share_of makes of that many keys, at most 16 to a CU.  (With 16 blocks at least
            // to a share, whatever the batch: one request of 4096 keys, 8 kv heads of 128, 39.7 us, 18.9 so; four 41.0,
            // 23.3; one of 131072 136, 120.)
            c.round = std::max(1, n_cu / heads_kv);
            const int64_t blocks = batch * ((keys + kFewKeys - 1) / kFewKeys + 1);
            const int64_t least = std::min<int64_t>(std::max<int64_t>(blocks / c.round, kFewestBlocks), kMostBlocks);
            c.shares = static_cast<int32_t>(std::min<int64_t>(16 * c.round, (blocks + least - 1) / least));
            c.grid = std::max(c.grid, static_cast<int64_t>(c.shares) * heads_kv);
            c.few_floats = 2 * static_cast<int64_t>(c.shares) * heads_kv * c.few_rows * (padded + 2);
        }
    }
    if (rows > 32) {
        c.tiles = static_cast<int32_t>((rows + kTileRows - 1) / kTileRows);
        // Two workgroups fit a CU.  A piece's rows cost a write and a read of their own, so there are no more
        // pieces than fill the CUs once (8 chunks of 512 tokens over 1k..8k, 8 kv heads, which fill them
        // twice: 320 us, in two pieces 476 us).
        // (a request's last tile may be empty in part; more than 256 requests' are not counted on the device)
        c.tile_count = batch * c.tiles;
        const bool counted = batch <= 256, mixed = counted && tokens < batch * max_q;
        if (counted) c.tile_count = std::min(c.tile_count, tokens * group / kTileRows + std::min(batch, tokens));
        const int64_t units = std::max<int64_t>(1, batch * heads_kv * c.tiles), slots = 2 * static_cast<int64_t>(n_cu);
        // Of a mixed batch most tiles hold nothing: there are about as many as its tokens fill, and one for every fourth
        // request (21 requests of 1 .. 88 tokens over 500 .. 9900, 16/4 heads of 80: 113 us counting all tiles, 86 us so).
        const int64_t held = std::max<int64_t>(1, mixed ? std::min(units, (tokens * group / kTileRows + (batch + 3) / 4) * heads_kv) : units);
        const int64_t splits = std::max<int64_t>(1, std::min((slots + held - 1) / held, (keys + 255) / 256));
        const int64_t each = ((keys + splits - 1) / splits + kKeyTile - 1) / kKeyTile * kKeyTile;
        c.split_keys = static_cast<int32_t>(each);
        c.splits = static_cast<int32_t>((keys + each - 1) / each);
        c.tile_floats = c.splits > 1 ? c.tile_count * heads_kv * c.splits * kTileRows * (padded + 2) : 0;
        const int64_t tiles = c.tile_count * heads_kv;
        c.grid = std::max(c.grid, tiles * c.splits);
        if (c.splits > 1) c.grid = std::max(c.grid, tiles * (kTileRows / join_rows(tiles)));
    }
    return c;
}

}  // namespace bsm_att
