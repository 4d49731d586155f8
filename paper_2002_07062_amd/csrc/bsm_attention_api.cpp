// C ABI of attention: argument checks, plans and launches.  Every failure is a status code plus a
// thread-local message; nothing is thrown across the ABI.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <array>
#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <memory>
#include <new>
#include <utility>
#include <vector>

#include "bsm.h"
#include "bsm_attention_plan.hpp"
#include "bsm_error.hpp"

struct bsm_attention_plan_s {
    int device = -1;  // -1: host-only plan
    bsm_schedule schedule = BSM_SCHED_RR;
    int n_xcd = 1;
    bsm_att::Sequences seqs;
    int32_t window = 0;  // as given
    int64_t n_forward = 0, n_q = 0, n_kv = 0, n_q_joins = 0, n_kv_joins = 0;
    int64_t q_part_rows = 0, kv_part_rows = 0;
    int32_t forward_rows = 0, dq_rows = 0, key_rows = 0;  // of a unit of the forward pass, of dq, of dk and dv
    bool few_units = false;                 // as in SequenceArgs
    void* d_units = nullptr;  // units of the forward pass, of dq, of dk and dv, and the joins of both
    std::atomic<bool> used{false};
};

namespace {

using bsm_att::Heads;
using bsm_att::kMostRows;

bsm_status fail(bsm_status st, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return bsm::report(st, buf);
}

bsm_status hip_fail(hipError_t e, const char* what) {
    return fail(BSM_ERR_HIP, "%s: %s (%d)", what, hipGetErrorString(e), static_cast<int>(e));
}

// Restores the caller's current device on scope exit.
struct DeviceGuard {
    int prev = -1;
    bool switched = false;
    hipError_t enter(int device) {
        hipError_t e = hipGetDevice(&prev);
        if (e != hipSuccess) return e;
        if (prev != device) {
            e = hipSetDevice(device);
            if (e != hipSuccess) return e;
            switched = true;
        }
        return hipSuccess;
    }
    ~DeviceGuard() {
        if (switched) (void)hipSetDevice(prev);
    }
};

constexpr int64_t kMostStride = int64_t{1} << 40;
constexpr int64_t kMostWorkgroups = (int64_t{1} << 24) - 1;  // of 256 threads: a launch has less than 2^32

bsm_status check_dims(int64_t heads_q, int64_t heads_kv, int64_t dim) {
    if (heads_q < 1 || heads_kv < 1 || heads_q % heads_kv != 0 || heads_q > 65535)
        return fail(BSM_ERR_INVALID_ARG, "heads_q %lld must be a multiple of heads_kv %lld, both in 1 .. 65535",
                    static_cast<long long>(heads_q), static_cast<long long>(heads_kv));
    if (dim < 1) return fail(BSM_ERR_INVALID_ARG, "head_dim %lld", static_cast<long long>(dim));
    if (dim % 8 != 0 || dim > 128)
        return fail(BSM_ERR_UNSUPPORTED, "head_dim %lld: a multiple of 8 up to 128 is supported", static_cast<long long>(dim));
    return BSM_OK;
}

bsm_status check_scale(float scale) {
    // (past 2^127 its product with log2(e) would be infinite, and a score of 0 NaN)
    if (!(scale > 0.0f) || !(scale <= 0x1p127f)) return fail(BSM_ERR_INVALID_ARG, "scale must be > 0 and at most 2^127");
    return BSM_OK;
}

// Bytes of memory that an operand spans.
struct Span {
    uintptr_t from = 0, to = 0;
};
bool overlap(const Span& a, const Span& b) { return a.from < b.to && b.from < a.to; }

// Rows of an operand: of every sequence b, [start[b], start[b] + len[b]).
struct Rows {
    const std::vector<int64_t>* start = nullptr;  // null: one sequence of rows 0 .. end - 1
    const std::vector<int32_t>* len = nullptr;
    int64_t end = 0, longest = 0;  // largest row + 1, rows of the longest sequence
    bool shared = false;           // two sequences have a row in common
    bool in_order = true;          // no sequence starts before the one before it
};

// Whether elements at sums of multiples of the strides, with `inner` contiguous ones at each, are apart.
bool nested(std::vector<std::pair<int64_t, int64_t>> stride_count, int64_t inner) {
    std::sort(stride_count.begin(), stride_count.end());
    for (const auto& [stride, count] : stride_count) {
        if (count <= 1) continue;
        if (stride < inner) return false;
        inner += stride * (count - 1);
    }
    return true;
}

// An operand with `heads` heads.  A written one must have a place of its own for each row.
bsm_status take(const char* name, const bsm_heads* h, const Rows& r, int64_t heads, int64_t dim, bool written, Heads* out, Span* span) {
    if (!h) return fail(BSM_ERR_INVALID_ARG, "%s is NULL", name);
    *span = {};
    *out = {static_cast<uint16_t*>(h->data), h->seq, h->row, h->head};
    if (h->seq < 0 || h->row < 0 || h->head < 0 || h->seq > kMostStride || h->row > kMostStride || h->head > kMostStride)
        return fail(BSM_ERR_INVALID_ARG, "%s: strides must be in 0 .. 2^40", name);
    if (r.end == 0) return BSM_OK;  // no rows
    if (!h->data) return fail(BSM_ERR_INVALID_ARG, "%s: data is NULL", name);
    if (reinterpret_cast<uintptr_t>(h->data) % 2 != 0)
        return fail(BSM_ERR_INVALID_ARG, "%s: data is not aligned to the element size", name);
    const int64_t batch = r.start ? static_cast<int64_t>(r.start->size()) : 1;
    const double far = static_cast<double>(batch) * h->seq + static_cast<double>(r.end) * h->row + static_cast<double>(heads) * h->head;
    if (far > 1.0e18) return fail(BSM_ERR_INVALID_ARG, "%s: rows too far apart", name);
    int64_t last = (r.end - 1) * h->row;  // of the rows' elements
    if (h->seq != 0 && r.start) {
        last = 0;
        for (int64_t b = 0; b < batch; ++b)
            if ((*r.len)[b] > 0) last = std::max(last, b * h->seq + ((*r.start)[b] + (*r.len)[b] - 1) * h->row);
    }
    span->from = reinterpret_cast<uintptr_t>(h->data);
    span->to = span->from + 2 * static_cast<uintptr_t>(last + (heads - 1) * h->head + dim);
    if (!written) return BSM_OK;
    // within a sequence: heads inside a row, or rows inside a head
    const int64_t rows = h->seq == 0 ? r.end : r.longest;
    const bool heads_inside = (heads == 1 || h->head >= dim) && (rows == 1 || h->row >= (heads - 1) * h->head + dim);
    const bool rows_inside = (rows == 1 || h->row >= dim) && (heads == 1 || h->head >= (rows - 1) * h->row + dim);
    bool apart = heads_inside || rows_inside;
    // between sequences: disjoint rows of one numbering, or blocks that follow each other (packed rows on
    // top of a sequence stride only move the sequences further apart)
    if (h->seq == 0) {
        apart = apart && !r.shared;
    } else if (batch > 1) {
        const int64_t block = (r.end - 1) * h->row + (heads - 1) * h->head + dim;
        const int64_t own = (r.longest - 1) * h->row + (heads - 1) * h->head + dim;
        apart = apart && (h->seq >= block || (r.in_order && h->seq >= own));
        // or sequences inside a row or a head, as where the rows or the heads come first
        apart = apart || nested({{h->seq, batch}, {h->row, r.end}, {h->head, heads}}, dim);
    }
    if (!apart) return fail(BSM_ERR_INVALID_ARG, "%s: rows overlap each other", name);
    return BSM_OK;
}

// How often an operand steps by a stride.
struct Axis {
    int64_t stride, count;
};
// Whether two operands, each of blocks of `dim` elements at sums of its axes' steps, are apart because they interleave:
// modulo one of the strides, which their larger strides are multiples of, they keep to different parts.
bool interleave(const uint16_t* x, const std::array<Axis, 3>& xs, const uint16_t* y, const std::array<Axis, 3>& ys, int64_t dim) {
    const auto part = [&](const std::array<Axis, 3>& axes, int64_t period) {  // elements of a period that may be used
        int64_t n = dim;
        for (const Axis& a : axes)
            if (a.stride % period != 0) n += a.stride * (a.count - 1);
        return n;
    };
    const int64_t bytes = static_cast<int64_t>(reinterpret_cast<uintptr_t>(y) - reinterpret_cast<uintptr_t>(x));
    for (const auto* axes : {&xs, &ys})
        for (const Axis& a : *axes) {
            if (a.stride < dim || a.count < 2) continue;
            const int64_t period = 2 * a.stride, at = (bytes % period + period) % period;  // of y behind x, in bytes
            if (at >= 2 * part(xs, a.stride) && at + 2 * part(ys, a.stride) <= period) return true;
        }
    return false;
}

// Whether two operands are apart sequence by sequence.
bool sequences_apart(const Heads& x, const Rows& xr, int64_t x_heads, const Heads& y, const Rows& yr, int64_t y_heads, int64_t dim) {
    struct Block {
        uintptr_t from, to;
        int of;
    };
    std::vector<Block> blocks;
    const auto add = [&](const Heads& t, const Rows& r, int64_t heads, int of) {
        for (size_t b = 0; b < r.start->size(); ++b) {
            if ((*r.len)[b] == 0) continue;
            const uintptr_t from = reinterpret_cast<uintptr_t>(t.p + static_cast<int64_t>(b) * t.seq + (*r.start)[b] * t.row);
            blocks.push_back({from, from + 2 * static_cast<uintptr_t>(((*r.len)[b] - 1) * t.row + (heads - 1) * t.head + dim), of});
        }
    };
    add(x, xr, x_heads, 0);
    add(y, yr, y_heads, 1);
    std::sort(blocks.begin(), blocks.end(), [](const Block& p, const Block& q) { return p.from < q.from; });
    uintptr_t end[2] = {0, 0};  // of the blocks so far
    for (const Block& b : blocks) {
        if (b.from < end[1 - b.of]) return false;
        end[b.of] = std::max(end[b.of], b.to);
    }
    return true;
}

// The same without sequences: rows are token indices.
bsm_status take_rows(const char* name, const bsm_heads* h, int64_t tokens, int64_t heads, int64_t dim, bool written, Heads* out,
                     Span* span) {
    if (!h) return fail(BSM_ERR_INVALID_ARG, "%s is NULL", name);
    const bsm_heads one = {h->data, 0, h->row, h->head};
    Rows r;
    r.end = r.longest = tokens;
    return take(name, &one, r, heads, dim, written, out, span);
}

Rows q_rows(const bsm_att::Sequences& s) { return {&s.q_start, &s.q_len, s.q_end, s.q_longest, s.q_shared, s.q_in_order}; }
Rows kv_rows(const bsm_att::Sequences& s) { return {&s.kv_start, &s.kv_len, s.kv_end, s.kv_longest, s.kv_shared, s.kv_in_order}; }

Span bytes_at(const void* p, int64_t bytes) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    return {a, a + static_cast<uintptr_t>(bytes)};
}

// Plan creation can be made to fail for tests of the failure paths, as every plan's.
bool fails(const char* how) {
    const char* v = std::getenv("BSM_TEST_ALLOC_FAIL");
    return v && std::strcmp(v, how) == 0;
}

bsm_status create(bsm_attention_plan* out_plan, const int32_t* q_len, const int32_t* kv_len, const int64_t* q_start,
                  const int64_t* kv_start, int64_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim, int32_t causal,
                  int32_t window, bsm_schedule schedule, const bsm_topology* topology, int device) {
    if (!out_plan) return fail(BSM_ERR_INVALID_ARG, "out_plan is NULL");
    *out_plan = nullptr;
    if (batch < 0 || batch > (int64_t{1} << 24)) return fail(BSM_ERR_INVALID_ARG, "batch %lld", static_cast<long long>(batch));
    if (batch > 0 && (!q_len || !kv_len)) return fail(BSM_ERR_INVALID_ARG, "q_len or kv_len is NULL");
    bsm_status st = check_dims(heads_q, heads_kv, head_dim);
    if (st != BSM_OK) return st;
    if (window < 0) return fail(BSM_ERR_INVALID_ARG, "window %d", window);
    if (window > 0 && !causal) return fail(BSM_ERR_INVALID_ARG, "a window needs causal");
    if (schedule != BSM_SCHED_RR && schedule != BSM_SCHED_BALANCED && schedule != BSM_SCHED_XCD)
        return fail(BSM_ERR_INVALID_ARG, "unknown schedule %d", static_cast<int>(schedule));
    if (device < -1) return fail(BSM_ERR_INVALID_ARG, "device %d", device);
    if (device == -1 && !topology) return fail(BSM_ERR_INVALID_ARG, "a host-only plan (device -1) needs a topology");
    int n_xcd = 8, n_cu = 256;
    if (device >= 0) {
        int n = 0;
        const hipError_t e = hipGetDeviceCount(&n);
        if (e != hipSuccess) return hip_fail(e, "hipGetDeviceCount");
        if (device >= n) return fail(BSM_ERR_INVALID_ARG, "device %d of %d", device, n);
        bsm_topology t;
        st = bsm_default_topology(device, &t);
        if (st != BSM_OK) return st;
        n_xcd = t.n_xcd;
        n_cu = t.n_cu;
    }
    if (topology) {
        if (topology->n_xcd < 0 || topology->n_xcd > BSM_MAX_XCD)
            return fail(BSM_ERR_INVALID_ARG, "topology: n_xcd %d", topology->n_xcd);
        if (topology->n_xcd > 0) n_xcd = topology->n_xcd;
        if (topology->n_cu < 0 || topology->n_cu > 65536) return fail(BSM_ERR_INVALID_ARG, "topology: n_cu %d", topology->n_cu);
        if (topology->n_cu > 0) n_cu = topology->n_cu;
    }
    for (int64_t b = 0; b < batch; ++b) {
        if (q_len[b] < 0 || kv_len[b] < 0 || q_len[b] > kMostRows || kv_len[b] > kMostRows)
            return fail(BSM_ERR_INVALID_ARG, "sequence %lld: lengths %d, %d must be in 0 .. 2^30", static_cast<long long>(b),
                        q_len[b], kv_len[b]);
        if ((q_start && (q_start[b] < 0 || q_start[b] > kMostStride)) || (kv_start && (kv_start[b] < 0 || kv_start[b] > kMostStride)))
            return fail(BSM_ERR_INVALID_ARG, "sequence %lld: first rows must be in 0 .. 2^40", static_cast<long long>(b));
    }
    std::unique_ptr<bsm_attention_plan_s> p(new (std::nothrow) bsm_attention_plan_s);
    if (!p) return fail(BSM_ERR_OOM, "plan allocation failed");
    try {
        bsm_att::Sequences& s = p->seqs;
        s.batch = batch;
        if (batch > 0) {
            s.q_len.assign(q_len, q_len + batch);
            s.kv_len.assign(kv_len, kv_len + batch);
        }
        s.heads_q = heads_q;
        s.heads_kv = heads_kv;
        s.dim = head_dim;
        s.mask = {causal ? 1 : 0, bsm_att::held_window(window)};
        p->window = window;
        bsm_att::finish_sequences(&s, q_start, kv_start);
        const double units = (static_cast<double>(s.total_q) / bsm_att::kTileRows + batch) * heads_q +
                             (static_cast<double>(s.total_kv) / bsm_att::kTileRows + batch) * heads_kv;
        if (units > kMostWorkgroups) return fail(BSM_ERR_INVALID_ARG, "too many rows for one plan");
        p->forward_rows = bsm_att::query_rows(s, n_cu);
        int64_t halves = 0;  // units of 64 rows, where there are such
        for (int64_t b = 0; b < batch; ++b) halves += (s.q_len[b] + p->forward_rows - 1) / p->forward_rows * int64_t{heads_q};
        p->few_units = halves <= 2 * static_cast<int64_t>(n_cu) && s.kv_longest > 64;
        // dq's units are the same, but of heads over 64 their halves need the registers of a whole CU
        const bool long_heads = bsm_att::padded_dim(s.dim) > 64;
        p->dq_rows = long_heads && halves > n_cu ? bsm_att::kTileRows : p->forward_rows;
        // workgroups on a CU: two, but of the gradient's kernels for longer heads one, except whole units of dq
        const int64_t cus = n_cu;
        const bool pairs = !long_heads || p->dq_rows == bsm_att::kTileRows;
        const bsm_att::Units f = bsm_att::make_units(s, false, p->forward_rows, 0, false, schedule, n_xcd);
        const bsm_att::Units q = bsm_att::make_units(s, false, p->dq_rows, pairs ? 2 * cus : cus, pairs, schedule, n_xcd);
        p->key_rows = bsm_att::key_rows(s, n_cu);
        const bsm_att::Units kv = bsm_att::make_units(s, true, p->key_rows, long_heads ? cus : 2 * cus, false, schedule, n_xcd);
        p->n_forward = static_cast<int64_t>(f.units.size());
        p->n_q = static_cast<int64_t>(q.units.size());
        p->n_kv = static_cast<int64_t>(kv.units.size());
        p->n_q_joins = static_cast<int64_t>(q.joins.size());
        p->n_kv_joins = static_cast<int64_t>(kv.joins.size());
        p->q_part_rows = q.part_rows;
        p->kv_part_rows = kv.part_rows;
        // (those of dk and dv of longer heads have 512 threads)
        if (std::max({p->n_forward, p->n_q, p->n_kv * (long_heads ? 2 : 1)}) > kMostWorkgroups) return fail(BSM_ERR_INVALID_ARG, "too many rows for one plan");
        p->device = device;
        p->schedule = schedule;
        p->n_xcd = n_xcd;
        if (fails("host")) throw std::bad_alloc();
        if (device >= 0 && p->n_q + p->n_kv > 0) {
            std::vector<bsm_att::Unit> table;
            for (const auto* units : {&f.units, &q.units, &kv.units, &q.joins, &kv.joins})
                table.insert(table.end(), units->begin(), units->end());
            DeviceGuard g;
            hipError_t e = g.enter(device);
            if (e != hipSuccess) return hip_fail(e, "hipSetDevice");
            const size_t bytes = table.size() * sizeof(bsm_att::Unit);
            e = fails("device") ? hipErrorOutOfMemory : hipMalloc(&p->d_units, bytes);
            if (e != hipSuccess) {
                (void)hipGetLastError();
                return fail(e == hipErrorOutOfMemory ? BSM_ERR_OOM : BSM_ERR_HIP, "hipMalloc(%zu) for the work table: %s", bytes,
                            hipGetErrorString(e));
            }
            e = hipMemcpy(p->d_units, table.data(), bytes, hipMemcpyHostToDevice);
            if (e != hipSuccess) {
                st = hip_fail(e, "uploading the work table");
                (void)hipFree(p->d_units);
                return st;
            }
        }
    } catch (const std::exception&) {
        return fail(BSM_ERR_OOM, "host allocation failed while planning");
    }
    *out_plan = p.release();
    return BSM_OK;
}

bsm_status check_plan(bsm_attention_plan p) {
    if (!p) return fail(BSM_ERR_INVALID_ARG, "plan is NULL");
    if (p->device < 0) return fail(BSM_ERR_UNSUPPORTED, "host-only plan (device -1) cannot execute");
    return BSM_OK;
}

bsm_status forward(bsm_attention_plan p, const bsm_heads* q, const bsm_heads* k, const bsm_heads* v, const bsm_heads* o, float* lse,
                   float scale, void* stream) {
    bsm_status st = check_plan(p);
    if (st != BSM_OK) return st;
    if ((st = check_scale(scale)) != BSM_OK) return st;
    const bsm_att::Sequences& s = p->seqs;
    const Rows qr = q_rows(s), kr = kv_rows(s);
    bsm_att::SequenceArgs a{};
    Span sq, sk, sv, so;
    if ((st = take("q", q, qr, s.heads_q, s.dim, false, &a.q, &sq)) != BSM_OK ||
        (st = take("k", k, kr, s.heads_kv, s.dim, false, &a.k, &sk)) != BSM_OK ||
        (st = take("v", v, kr, s.heads_kv, s.dim, false, &a.v, &sv)) != BSM_OK ||
        (st = take("o", o, qr, s.heads_q, s.dim, true, &a.o, &so)) != BSM_OK)
        return st;
    const Span sl = lse ? bytes_at(lse, 4 * s.heads_q * s.total_q) : Span{};
    if (overlap(so, sq) || overlap(so, sk) || overlap(so, sv)) return fail(BSM_ERR_ALIAS, "o overlaps an operand");
    if (overlap(sl, sq) || overlap(sl, sk) || overlap(sl, sv) || overlap(sl, so)) return fail(BSM_ERR_ALIAS, "lse overlaps an operand");
    if (reinterpret_cast<uintptr_t>(lse) % 4 != 0) return fail(BSM_ERR_INVALID_ARG, "lse is not aligned to its element size");
    if (p->n_forward == 0) return BSM_OK;
    a.lse = lse;
    a.total_q = s.total_q;
    a.group = s.heads_q / s.heads_kv;
    a.dim = s.dim;
    a.unit_rows = p->forward_rows;
    a.few_units = p->few_units;
    a.mask = s.mask;
    a.scale = scale;
    DeviceGuard g;
    hipError_t e = g.enter(p->device);
    if (e != hipSuccess) return hip_fail(e, "hipSetDevice");
    e = bsm_att::launch_attention(a, static_cast<const bsm_att::Unit*>(p->d_units), p->n_forward, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "kernel launch");
    p->used = true;
    return BSM_OK;
}

// The workspace: delta of every query row and head, and the parts of dk and dv, and of dq.
int64_t delta_bytes(const bsm_att::Sequences& s) { return (4 * s.heads_q * s.total_q + 15) / 16 * 16; }
int64_t workspace_of(bsm_attention_plan p) {
    return delta_bytes(p->seqs) + 4 * (2 * p->kv_part_rows + p->q_part_rows) * bsm_att::padded_dim(p->seqs.dim);
}

bsm_status backward(bsm_attention_plan p, const bsm_heads* q, const bsm_heads* k, const bsm_heads* v, const bsm_heads* o,
                    const float* lse, const bsm_heads* dout, const bsm_heads* dq, const bsm_heads* dk, const bsm_heads* dv, float scale,
                    void* workspace, int64_t workspace_bytes, void* stream) {
    bsm_status st = check_plan(p);
    if (st != BSM_OK) return st;
    if ((st = check_scale(scale)) != BSM_OK) return st;
    const bsm_att::Sequences& s = p->seqs;
    const Rows qr = q_rows(s), kr = kv_rows(s);
    bsm_att::SequenceArgs a{};
    Span in[7], out[4];
    if ((st = take("q", q, qr, s.heads_q, s.dim, false, &a.q, &in[0])) != BSM_OK ||
        (st = take("k", k, kr, s.heads_kv, s.dim, false, &a.k, &in[1])) != BSM_OK ||
        (st = take("v", v, kr, s.heads_kv, s.dim, false, &a.v, &in[2])) != BSM_OK ||
        (st = take("o", o, qr, s.heads_q, s.dim, false, &a.o, &in[3])) != BSM_OK ||
        (st = take("dout", dout, qr, s.heads_q, s.dim, false, &a.dout, &in[4])) != BSM_OK ||
        (st = take("dq", dq, qr, s.heads_q, s.dim, true, &a.dq, &out[0])) != BSM_OK ||
        (st = take("dk", dk, kr, s.heads_kv, s.dim, true, &a.dk, &out[1])) != BSM_OK ||
        (st = take("dv", dv, kr, s.heads_kv, s.dim, true, &a.dv, &out[2])) != BSM_OK)
        return st;
    const int64_t need = workspace_of(p), lse_bytes = 4 * s.heads_q * s.total_q;
    if ((lse_bytes > 0 && !lse) || (need > 0 && !workspace)) return fail(BSM_ERR_INVALID_ARG, "lse or workspace is NULL");
    if (workspace_bytes < need)
        return fail(BSM_ERR_INVALID_ARG, "workspace of %lld bytes, %lld needed", static_cast<long long>(workspace_bytes),
                    static_cast<long long>(need));
    if (reinterpret_cast<uintptr_t>(lse) % 4 != 0) return fail(BSM_ERR_INVALID_ARG, "lse is not aligned to its element size");
    if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return fail(BSM_ERR_INVALID_ARG, "workspace is not aligned to 16 bytes");
    in[5] = bytes_at(lse, lse_bytes);
    out[3] = bytes_at(workspace, need);
    in[6] = {};
    for (const Span& x : out)
        for (const Span& y : in)
            if (overlap(x, y)) return fail(BSM_ERR_ALIAS, "a gradient or the workspace overlaps an operand");
    for (int i = 0; i < 3; ++i) {
        if (overlap(out[i], out[3])) return fail(BSM_ERR_ALIAS, "a gradient overlaps the workspace");
    }
    const struct {
        const Heads& t;
        const Rows& r;
        int64_t heads;
    } grads[3] = {{a.dq, qr, s.heads_q}, {a.dk, kr, s.heads_kv}, {a.dv, kr, s.heads_kv}};
    for (int i = 0; i < 3; ++i)
        for (int j = 0; j < i; ++j) {
            if (!overlap(out[i], out[j])) continue;
            const auto &x = grads[j], &y = grads[i];
            const auto axes = [&](const auto& g) {
                return std::array<Axis, 3>{{{g.t.seq, s.batch}, {g.t.row, g.r.end}, {g.t.head, g.heads}}};
            };
            if (!interleave(x.t.p, axes(x), y.t.p, axes(y), s.dim) && !sequences_apart(x.t, x.r, x.heads, y.t, y.r, y.heads, s.dim))
                return fail(BSM_ERR_ALIAS, "two gradients overlap");
        }
    a.lse = const_cast<float*>(lse);
    a.delta = static_cast<float*>(workspace);
    a.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + delta_bytes(s));
    a.dq_part = a.part + 2 * p->kv_part_rows * bsm_att::padded_dim(s.dim);
    a.total_q = s.total_q;
    a.group = s.heads_q / s.heads_kv;
    a.dim = s.dim;
    a.unit_rows = p->dq_rows;
    a.key_rows = p->key_rows;
    a.few_units = p->few_units;
    a.mask = s.mask;
    a.scale = scale;
    if (p->n_q + p->n_kv == 0) return BSM_OK;
    DeviceGuard g;
    hipError_t e = g.enter(p->device);
    if (e != hipSuccess) return hip_fail(e, "hipSetDevice");
    bsm_att::GradientUnits u{};
    u.q = static_cast<const bsm_att::Unit*>(p->d_units) + p->n_forward;
    u.kv = u.q + p->n_q;
    u.joins = u.kv + p->n_kv;
    u.n_q = p->n_q;
    u.n_kv = p->n_kv;
    u.n_q_joins = p->n_q_joins;
    u.n_kv_joins = p->n_kv_joins;
    e = bsm_att::launch_attention_backward(a, u, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "kernel launch");
    p->used = true;
    return BSM_OK;
}

// -------------------------------------------------------------------------------- paged cache
bsm_status take_cache(const bsm_cache* c, bsm_att::Cache* out, Span* k, Span* v) {
    if (!c) return fail(BSM_ERR_INVALID_ARG, "cache is NULL");
    bsm_status st = check_dims(c->heads, c->heads, c->head_dim);
    if (st != BSM_OK) return st;
    if (c->n_pages < 0 || c->n_pages > 0x7FFFFFFF || c->page_size < 1)
        return fail(BSM_ERR_INVALID_ARG, "cache: %lld pages of %d tokens", static_cast<long long>(c->n_pages), c->page_size);
    if (c->page_stride < 0 || c->row_stride < 0 || c->head_stride < 0 || c->page_stride > kMostStride || c->row_stride > kMostStride ||
        c->head_stride > kMostStride)
        return fail(BSM_ERR_INVALID_ARG, "cache: strides must be in 0 .. 2^40");
    *out = {static_cast<uint16_t*>(c->k), static_cast<uint16_t*>(c->v), c->page_stride, c->row_stride, c->head_stride, c->n_pages,
            c->page_size, c->heads, c->head_dim};
    *k = *v = {};
    if (c->n_pages == 0) return BSM_OK;
    if (!c->k || !c->v) return fail(BSM_ERR_INVALID_ARG, "cache: k or v is NULL");
    if ((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v)) % 2 != 0)
        return fail(BSM_ERR_INVALID_ARG, "cache: k or v is not aligned to the element size");
    const double far = static_cast<double>(c->n_pages) * c->page_stride + static_cast<double>(c->page_size) * c->row_stride +
                       static_cast<double>(c->heads) * c->head_stride;
    if (far > 1.0e18) return fail(BSM_ERR_INVALID_ARG, "cache: pages too far apart");
    const int64_t elems = (c->n_pages - 1) * c->page_stride + (c->page_size - 1) * c->row_stride + (c->heads - 1) * c->head_stride +
                          c->head_dim;
    *k = bytes_at(c->k, 2 * elems);
    *v = bytes_at(c->v, 2 * elems);
    return BSM_OK;
}

hipError_t compute_units(int device, int* n) { return hipDeviceGetAttribute(n, hipDeviceAttributeMultiprocessorCount, device); }

bsm_status check_paged_sizes(int64_t batch, int64_t tokens, int64_t heads_q, int64_t heads_kv, int64_t dim, int64_t max_q,
                             int64_t max_kv) {
    bsm_status st = check_dims(heads_q, heads_kv, dim);
    if (st != BSM_OK) return st;
    if (batch < 0 || tokens < 0 || max_q < 0 || max_kv < 0 || batch > (int64_t{1} << 24) || tokens > kMostRows || max_kv > kMostRows)
        return fail(BSM_ERR_INVALID_ARG, "batch %lld, tokens %lld, max_q %lld, max_kv %lld", static_cast<long long>(batch),
                    static_cast<long long>(tokens), static_cast<long long>(max_q), static_cast<long long>(max_kv));
    if (static_cast<double>(std::min(max_q, tokens)) * (static_cast<double>(heads_q) / heads_kv) > kMostRows)
        return fail(BSM_ERR_INVALID_ARG, "max_q %lld is too large", static_cast<long long>(max_q));
    return BSM_OK;
}

bsm_status paged_cut(int64_t batch, int64_t tokens, int32_t heads_q, int32_t heads_kv, int32_t dim, int32_t max_q, int32_t max_kv,
                     int n_cu, bsm_att::PagedCut* cut) {
    *cut = bsm_att::cut_paged(batch, tokens, heads_kv, heads_q / heads_kv, dim, max_q, max_kv, n_cu);
    if (cut->grid > kMostWorkgroups)
        return fail(BSM_ERR_INVALID_ARG, "batch %lld with max_q %d is too large for one call", static_cast<long long>(batch), max_q);
    return BSM_OK;
}

bsm_status paged(const bsm_cache* cache, const bsm_heads* q, const bsm_heads* o, const int32_t* table, int32_t width,
                 const int32_t* q_start, const int32_t* kv_len, int64_t batch, int64_t tokens, int32_t heads_q, int32_t max_q,
                 int32_t max_kv, int32_t window, float scale, void* workspace, int64_t workspace_bytes, void* stream) {
    bsm_att::PagedArgs a{};
    Span sk, sv, sq, so;
    bsm_status st = take_cache(cache, &a.cache, &sk, &sv);
    if (st != BSM_OK) return st;
    if (width < 0 || window < 0) return fail(BSM_ERR_INVALID_ARG, "width %d, window %d", width, window);
    if (static_cast<int64_t>(width) * cache->page_size > kMostRows)
        return fail(BSM_ERR_INVALID_ARG, "width %d: more than 2^30 tokens", width);
    if ((st = check_scale(scale)) != BSM_OK) return st;
    if (max_kv == 0) max_kv = width * cache->page_size;
    if ((st = check_paged_sizes(batch, tokens, heads_q, cache->heads, cache->head_dim, max_q, max_kv)) != BSM_OK) return st;
    if ((st = take_rows("q", q, tokens, heads_q, cache->head_dim, false, &a.q, &sq)) != BSM_OK ||
        (st = take_rows("o", o, tokens, heads_q, cache->head_dim, true, &a.o, &so)) != BSM_OK)
        return st;
    if (overlap(so, sq) || overlap(so, sk) || overlap(so, sv)) return fail(BSM_ERR_ALIAS, "o overlaps an operand");
    if (batch == 0 || tokens == 0 || max_q == 0) return BSM_OK;
    if (!q_start || !kv_len || (!table && width > 0)) return fail(BSM_ERR_INVALID_ARG, "table, q_start or kv_len is NULL");
    if ((reinterpret_cast<uintptr_t>(table) | reinterpret_cast<uintptr_t>(q_start) | reinterpret_cast<uintptr_t>(kv_len)) % 4 != 0)
        return fail(BSM_ERR_INVALID_ARG, "table, q_start or kv_len is not aligned to its element size");
    if (overlap(so, bytes_at(table, 4 * batch * width)) || overlap(so, bytes_at(q_start, 4 * batch + 4)) ||
        overlap(so, bytes_at(kv_len, 4 * batch)))
        return fail(BSM_ERR_ALIAS, "o overlaps an operand");
    int device = 0, n_cu = 0;
    hipError_t e = hipGetDevice(&device);
    if (e == hipSuccess) e = compute_units(device, &n_cu);
    if (e != hipSuccess) return hip_fail(e, "device query");
    bsm_att::PagedCut cut;
    if ((st = paged_cut(batch, tokens, heads_q, cache->heads, cache->head_dim, max_q, max_kv, n_cu, &cut)) != BSM_OK) return st;
    const int64_t need = 4 * (cut.few_floats + cut.tile_floats);
    if (workspace_bytes < need || (need > 0 && !workspace))
        return fail(BSM_ERR_INVALID_ARG, "workspace of %lld bytes, %lld needed", static_cast<long long>(workspace_bytes),
                    static_cast<long long>(need));
    if (need > 0) {
        const Span w = bytes_at(workspace, need);
        if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return fail(BSM_ERR_INVALID_ARG, "workspace is not aligned to 16 bytes");
        if (overlap(w, sq) || overlap(w, so) || overlap(w, sk) || overlap(w, sv) || overlap(w, bytes_at(table, 4 * batch * width)) ||
            overlap(w, bytes_at(q_start, 4 * batch + 4)) || overlap(w, bytes_at(kv_len, 4 * batch)))
            return fail(BSM_ERR_ALIAS, "the workspace overlaps an operand");
    }
    a.table = table;
    a.q_start = q_start;
    a.kv_len = kv_len;
    a.batch = batch;
    a.tokens = tokens;
    a.width = width;
    a.max_q = max_q;
    a.group = heads_q / cache->heads;
    a.window = bsm_att::held_window(window);
    a.scale = scale;
    a.few_rows = cut.few_rows;
    a.shares = cut.shares;
    a.round = cut.round;
    a.tiles = cut.tiles;
    a.tile_count = cut.tile_count;
    a.splits = cut.splits;
    a.split_keys = cut.split_keys;
    a.few_part = static_cast<float*>(workspace);
    a.tile_part = a.few_part + cut.few_floats;
    e = bsm_att::launch_attention_paged(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "kernel launch");
    return BSM_OK;
}

bsm_status slots_of(const int32_t* cached, const int32_t* fresh, int64_t batch, int32_t page_size, int64_t n_pages, int32_t* table,
                    int32_t width, const int32_t* free_pages, int64_t free_cap, const int32_t* n_free, int32_t* q_start, int32_t* kv_len,
                    int64_t* slots, int64_t n_slots, int32_t* taken, void* stream) {
    if (batch < 0 || batch > (int64_t{1} << 24) || page_size < 1 || n_pages < 0 || n_pages > 0x7FFFFFFF || width < 0 || free_cap < 0 ||
        n_slots < 0 || n_slots > kMostRows)
        return fail(BSM_ERR_INVALID_ARG, "batch %lld, page_size %d, n_pages %lld, width %d, free_cap %lld, n_slots %lld",
                    static_cast<long long>(batch), page_size, static_cast<long long>(n_pages), width, static_cast<long long>(free_cap),
                    static_cast<long long>(n_slots));
    if (static_cast<int64_t>(width) * page_size > kMostRows) return fail(BSM_ERR_INVALID_ARG, "width %d: more than 2^30 tokens", width);
    if (!q_start || !taken || !n_free || (batch > 0 && (!cached || !fresh || !kv_len)) || (batch > 0 && width > 0 && !table) ||
        (free_cap > 0 && !free_pages) || (n_slots > 0 && !slots))
        return fail(BSM_ERR_INVALID_ARG, "an array is NULL");
    const Span in[4] = {bytes_at(cached, 4 * batch), bytes_at(fresh, 4 * batch), bytes_at(free_pages, 4 * free_cap), bytes_at(n_free, 4)};
    const Span out[5] = {bytes_at(table, 4 * batch * width), bytes_at(q_start, 4 * batch + 4), bytes_at(kv_len, 4 * batch),
                         bytes_at(slots, 8 * n_slots), bytes_at(taken, 8)};
    for (int i = 0; i < 5; ++i) {
        if (out[i].from % (i == 3 ? 8 : 4) != 0) return fail(BSM_ERR_INVALID_ARG, "an array is not aligned to its element size");
        for (const Span& x : in)
            if (overlap(out[i], x)) return fail(BSM_ERR_ALIAS, "an output overlaps an input");
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return fail(BSM_ERR_ALIAS, "two outputs overlap");
    }
    for (const Span& x : in)
        if (x.from % 4 != 0) return fail(BSM_ERR_INVALID_ARG, "an array is not aligned to its element size");
    int device = 0, n_cu = 0;
    hipError_t e = hipGetDevice(&device);
    if (e == hipSuccess) e = compute_units(device, &n_cu);
    if (e != hipSuccess) return hip_fail(e, "device query");
    const bsm_att::SlotArgs a = {cached, fresh, batch, page_size, width, n_pages, table, free_pages,
                                 free_cap, n_free, q_start, kv_len, slots, n_slots, taken};
    e = bsm_att::launch_cache_slots(a, n_cu, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "kernel launch");
    return BSM_OK;
}

bsm_status append(const bsm_cache* cache, const bsm_heads* k, const bsm_heads* v, const int64_t* slots, int64_t tokens, void* stream) {
    bsm_att::Cache c;
    Span sk, sv, fk, fv;
    Heads hk, hv;
    bsm_status st = take_cache(cache, &c, &sk, &sv);
    if (st != BSM_OK) return st;
    if (tokens < 0 || tokens > kMostRows) return fail(BSM_ERR_INVALID_ARG, "tokens %lld", static_cast<long long>(tokens));
    if ((st = take_rows("k", k, tokens, cache->heads, cache->head_dim, false, &hk, &fk)) != BSM_OK ||
        (st = take_rows("v", v, tokens, cache->heads, cache->head_dim, false, &hv, &fv)) != BSM_OK)
        return st;
    if (tokens == 0 || cache->n_pages == 0) return BSM_OK;
    if (!nested({{c.page, c.n_pages}, {c.row, c.page_size}, {c.head, c.heads}}, c.dim))
        return fail(BSM_ERR_INVALID_ARG, "cache: rows overlap each other");
    if (!slots) return fail(BSM_ERR_INVALID_ARG, "slots is NULL");
    if (reinterpret_cast<uintptr_t>(slots) % 8 != 0) return fail(BSM_ERR_INVALID_ARG, "slots is not aligned to its element size");
    const Span ss = bytes_at(slots, 8 * tokens);
    if (sk.from == sv.from) return fail(BSM_ERR_ALIAS, "the cache's k and v have the same place");
    const std::array<Axis, 3> axes = {{{c.page, c.n_pages}, {c.row, c.page_size}, {c.head, c.heads}}};
    if (overlap(sk, sv) && !interleave(c.k, axes, c.v, axes, c.dim)) return fail(BSM_ERR_ALIAS, "the cache's k and v overlap");
    if (overlap(sk, fk) || overlap(sk, fv) || overlap(sv, fk) || overlap(sv, fv) || overlap(sk, ss) || overlap(sv, ss))
        return fail(BSM_ERR_ALIAS, "the cache overlaps an operand");
    int device = 0, n_cu = 0;
    hipError_t e = hipGetDevice(&device);
    if (e == hipSuccess) e = compute_units(device, &n_cu);
    if (e != hipSuccess) return hip_fail(e, "device query");
    e = bsm_att::launch_cache_append(c, hk, hv, slots, tokens, n_cu, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "kernel launch");
    return BSM_OK;
}

// Nothing leaves the ABI as an exception (the checks' small vectors can fail to allocate).
template <class F>
bsm_status guarded(F&& f) {
    try {
        return f();
    } catch (const std::exception&) {
        return bsm::report(BSM_ERR_OOM, "host allocation failed");
    }
}

}  // namespace

extern "C" {

bsm_status bsm_attention_plan_create(bsm_attention_plan* out_plan, const int32_t* q_len, const int32_t* kv_len, const int64_t* q_start,
                                     const int64_t* kv_start, int64_t batch, int32_t heads_q, int32_t heads_kv, int32_t head_dim,
                                     int32_t causal, int32_t window, bsm_schedule schedule, const bsm_topology* topology, int device) {
    return guarded([&] {
        return create(out_plan, q_len, kv_len, q_start, kv_start, batch, heads_q, heads_kv, head_dim, causal, window, schedule, topology,
                      device);
    });
}

bsm_status bsm_attention_plan_describe(bsm_attention_plan plan, bsm_attention_stats* stats) {
    if (!plan || !stats) return fail(BSM_ERR_INVALID_ARG, "plan or stats is NULL");
    const bsm_att::Sequences& s = plan->seqs;
    *stats = {};
    stats->batch = s.batch;
    stats->total_q = s.total_q;
    stats->total_kv = s.total_kv;
    stats->q_units = plan->n_forward;
    stats->kv_units = plan->n_kv;
    stats->lse_elems = s.heads_q * s.total_q;
    stats->workspace_bytes = workspace_of(plan);
    stats->pairs = s.pairs;
    stats->heads_q = s.heads_q;
    stats->heads_kv = s.heads_kv;
    stats->head_dim = s.dim;
    stats->causal = s.mask.causal;
    stats->window = plan->window;
    stats->schedule = plan->schedule;
    stats->n_xcd = plan->n_xcd;
    const bool half_forward = plan->forward_rows < bsm_att::kTileRows, half_dq = plan->dq_rows < bsm_att::kTileRows;
    const bool long_steps = plan->few_units && bsm_att::padded_dim(s.dim) == 64;
    stats->forms = (half_forward ? BSM_ATTENTION_HALF_FORWARD : 0) | (half_dq ? BSM_ATTENTION_HALF_DQ : 0) |
                   (plan->key_rows < bsm_att::kTileRows ? BSM_ATTENTION_HALF_KEYS : 0) |
                   (long_steps && (half_forward || half_dq) ? BSM_ATTENTION_LONG_STEPS : 0) |
                   (plan->n_q_joins > 0 ? BSM_ATTENTION_DQ_PARTS : 0) | (plan->n_kv_joins > 0 ? BSM_ATTENTION_KEY_PARTS : 0);
    return BSM_OK;
}

bsm_status bsm_attention_plan_destroy(bsm_attention_plan plan) {
    if (!plan) return fail(BSM_ERR_INVALID_ARG, "plan is NULL");
    if (plan->d_units) {
        DeviceGuard g;
        if (g.enter(plan->device) == hipSuccess) {
            if (plan->used) (void)hipDeviceSynchronize();
            (void)hipFree(plan->d_units);
        }
    }
    delete plan;
    return BSM_OK;
}

bsm_status bsm_attention_execute(bsm_attention_plan plan, const bsm_heads* q, const bsm_heads* k, const bsm_heads* v, const bsm_heads* o,
                                 float* lse, float scale, void* stream) {
    return guarded([&] { return forward(plan, q, k, v, o, lse, scale, stream); });
}

bsm_status bsm_attention_backward(bsm_attention_plan plan, const bsm_heads* q, const bsm_heads* k, const bsm_heads* v,
                                  const bsm_heads* o, const float* lse, const bsm_heads* dout, const bsm_heads* dq, const bsm_heads* dk,
                                  const bsm_heads* dv, float scale, void* workspace, int64_t workspace_bytes, void* stream) {
    return guarded([&] { return backward(plan, q, k, v, o, lse, dout, dq, dk, dv, scale, workspace, workspace_bytes, stream); });
}

bsm_status bsm_cache_slots(const int32_t* cached, const int32_t* fresh, int64_t batch, int32_t page_size, int64_t n_pages, int32_t* table,
                           int32_t width, const int32_t* free_pages, int64_t free_cap, const int32_t* n_free, int32_t* q_start,
                           int32_t* kv_len, int64_t* slots, int64_t n_slots, int32_t* taken, void* stream) {
    return guarded([&] {
        return slots_of(cached, fresh, batch, page_size, n_pages, table, width, free_pages, free_cap, n_free, q_start, kv_len, slots,
                        n_slots, taken, stream);
    });
}

bsm_status bsm_cache_append(const bsm_cache* cache, const bsm_heads* k, const bsm_heads* v, const int64_t* slots, int64_t tokens,
                            void* stream) {
    return guarded([&] { return append(cache, k, v, slots, tokens, stream); });
}

bsm_status bsm_attention_paged(const bsm_cache* cache, const bsm_heads* q, const bsm_heads* o, const int32_t* table, int32_t width,
                               const int32_t* q_start, const int32_t* kv_len, int64_t batch, int64_t tokens, int32_t heads_q,
                               int32_t max_q, int32_t max_kv, int32_t window, float scale, void* workspace, int64_t workspace_bytes,
                               void* stream) {
    return guarded([&] {
        return paged(cache, q, o, table, width, q_start, kv_len, batch, tokens, heads_q, max_q, max_kv, window, scale, workspace,
                     workspace_bytes, stream);
    });
}

bsm_status bsm_attention_paged_workspace(int64_t batch, int64_t tokens, int32_t heads_q, int32_t heads_kv, int32_t head_dim, int32_t max_q,
                                         int32_t max_kv, int device, int64_t* bytes) {
    if (!bytes) return fail(BSM_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = 0;
    bsm_status st = check_paged_sizes(batch, tokens, heads_q, heads_kv, head_dim, max_q, max_kv);
    if (st != BSM_OK) return st;
    if (device < 0) return fail(BSM_ERR_INVALID_ARG, "device %d", device);
    int n = 0, n_cu = 0;
    hipError_t e = hipGetDeviceCount(&n);
    if (e != hipSuccess) return hip_fail(e, "hipGetDeviceCount");
    if (device >= n) return fail(BSM_ERR_INVALID_ARG, "device %d of %d", device, n);
    e = compute_units(device, &n_cu);
    if (e != hipSuccess) return hip_fail(e, "device query");
    bsm_att::PagedCut cut;
    if ((st = paged_cut(batch, tokens, heads_q, heads_kv, head_dim, max_q, max_kv, n_cu, &cut)) != BSM_OK) return st;
    *bytes = 4 * (cut.few_floats + cut.tile_floats);
    return BSM_OK;
}

}  // extern "C"
