// Work lists of attention over spans of a plan's batch: a window with sinks (tc_plan_set_window), sequences that share their first tokens (tc_plan_set_shared).
// Host code; the kernels are in tc_span.hip.
#include <algorithm>
#include <chrono>
#include <cstring>
#include <numeric>

#include "tc_internal.h"

namespace tc {

namespace {

tc_status fail(tc_status s, const char *msg) {
    set_error(msg);
    return s;
}

constexpr int kTilePages = kPrefillTileTokens / kBlock;
constexpr int kMinSweepTiles = 4;   // a piece of a cut sweep is not shorter than this
constexpr int kMinWavePages = 4;    // nor does a wave get fewer pages of a decode item that is shared out
constexpr int64_t kDecodeWaveSlots = (int64_t)kNumCu * kDecodeWgPerCu * kDecodeWaves;  // waves of decode-only workgroups that the chip holds
// Rates that the two branches are balanced with where a batch has both (one MI355X): what a sweep of 256 rows takes for a tile, and what a compute unit streams.
constexpr double kSweepTileUs = 1.8, kStreamCuBytesPerUs = 25e3;

int tiles_of(const SpanRuns &r) { return (r.pages() + kTilePages - 1) / kTilePages; }

// Rows of one sequence (or, with `from` >= 0 and runs given by the caller, of several) in blocks that a workgroup sweeps.
void add_blocks(const tc_plan *p, SpanList &s, int seq, int from) {
    const int per = kPrefillRows / p->G, q = p->q_start[seq + 1] - p->q_start[seq];
    for (int i = 0; i < q; i += per) {
        SpanBlock b;
        b.npos = std::min(per, q - i);
        b.qrow = p->q_start[seq] + i;
        b.pos = p->ctx_len[seq] + i;
        b.page_off = p->page_off[seq];
        b.runs = SpanRuns::of(b.pos, b.npos, s.window, s.sinks, from);
        b.partial = from > 0;
        s.blocks.push_back(b);
    }
}
void add_decode(const tc_plan *p, SpanList &s, int seq, int from) {
    SpanEntry e;
    e.qrow = p->q_start[seq];
    e.cols = p->G;
    e.pos = p->ctx_len[seq];
    e.page_off = p->page_off[seq];
    e.runs = SpanRuns::of(e.pos, 1, s.window, s.sinks, from);
    e.partial = from > 0;
    s.entries.push_back(e);
}
void add_sequence(const tc_plan *p, SpanList &s, int seq, int from) {
    if (p->q_start[seq + 1] - p->q_start[seq] == 1) add_decode(p, s, seq, from);
    else add_blocks(p, s, seq, from);
}

// The pieces of the sweeps and the waves of the decode items.
void share_out(const tc_plan *p, SpanList &s) {
    const int64_t Hkv = p->Hkv;
    int64_t tiles = 0, longest = 1, pages = 0;
    for (const SpanBlock &b : s.blocks) {
        tiles += tiles_of(b.runs);
        longest = std::max<int64_t>(longest, tiles_of(b.runs));
    }
    for (const SpanEntry &e : s.entries) pages += e.runs.pages();
    if (!s.blocks.empty() && (int64_t)s.blocks.size() * Hkv < kNumCu) {
        // Few sweeps: cut, so that they take the compute units that decodes beside them leave, all of them where there are none.
        int64_t target = kNumCu;
        if (pages > 0) {
            const double sweep_us = (double)tiles * Hkv * kSweepTileUs * p->D / 128, stream_us = (double)pages * Hkv * kBlock * p->token_bytes() / kStreamCuBytesPerUs;
            target = std::max<int64_t>((int64_t)s.blocks.size() * Hkv, (int64_t)(kNumCu * sweep_us / (sweep_us + stream_us)));
        }
        int64_t length = std::max<int64_t>(kMinSweepTiles, tiles * Hkv / std::max<int64_t>(target, 1));
        for (; length < longest; length++) {
            int64_t n = 0;
            for (const SpanBlock &b : s.blocks) n += (tiles_of(b.runs) + length - 1) / length;
            if (n * Hkv <= target) break;
        }
        for (SpanBlock &b : s.blocks) b.k = (int32_t)std::max<int64_t>(1, (tiles_of(b.runs) + length - 1) / length);
    }
    const bool sweeps = !s.blocks.empty();
    const int waves = sweeps ? kMixedWaves : kDecodeWaves;
    const int64_t slots = sweeps ? (int64_t)kNumCu * kMixedWaves : kDecodeWaveSlots;
    const int64_t per_wave = std::min<int64_t>(kMaxSplitPages, std::max<int64_t>(kMinWavePages, (pages * Hkv + slots - 1) / slots));
    s.waves_log2 = 0;
    if (!s.entries.empty()) {
        const int64_t mean = (pages + (int64_t)s.entries.size() - 1) / (int64_t)s.entries.size();
        while ((1 << s.waves_log2) < waves && ((int64_t)per_wave << s.waves_log2) < mean) s.waves_log2++;
    }
    s.wide = !sweeps && (pages * Hkv + per_wave - 1) / per_wave <= (int64_t)kNumCu * 2 * kDecodeWaves;
    // An item that is a little longer than the mean is not cut for it.
    const int64_t most = std::min<int64_t>((int64_t)kMaxSplitPages << s.waves_log2, (int64_t)(per_wave + per_wave / 2) << s.waves_log2);
    for (SpanEntry &e : s.entries) e.units = (int32_t)((e.runs.pages() + most - 1) / most);
}

bool fits(int64_t rows) { return rows < (int64_t)1 << 31; }

// Places of the partial results, records, decode items.
tc_status lay_out(const tc_plan *p, SpanList &s) {
    const int Hkv = p->Hkv, G = p->G;
    int64_t rows = 0, pieces = 0, units = 0;
    s.max_cols = 1;
    for (SpanBlock &b : s.blocks) {
        pieces += b.k;
        if (b.k == 1 && !b.partial) continue;
        b.row0 = rows;
        b.kv_rows = (int64_t)b.k * b.npos * G;
        rows += b.kv_rows * Hkv;
    }
    for (SpanEntry &e : s.entries) {
        units += e.units;
        s.max_cols = std::max(s.max_cols, (int)e.cols);
        if (e.units == 1 && !e.partial) continue;
        e.row0 = rows;
        rows += (int64_t)e.units * e.cols * Hkv;
    }
    if (!fits(rows) || !fits(pieces * Hkv) || !fits(units * Hkv)) return fail(TC_ERR_SPAN, "the batch has more partial results than 2^31 rows");
    s.n_rows = rows;

    // sweeps, the longest first
    s.order.resize(s.blocks.size());
    std::iota(s.order.begin(), s.order.end(), 0);
    std::stable_sort(s.order.begin(), s.order.end(), [&](int x, int y) {
        return (tiles_of(s.blocks[x].runs) + s.blocks[x].k - 1) / s.blocks[x].k > (tiles_of(s.blocks[y].runs) + s.blocks[y].k - 1) / s.blocks[y].k;
    });
    s.records.assign((size_t)pieces * kRecordInts, 0);
    int32_t *r = s.records.data();
    for (const int i : s.order) {
        const SpanBlock &b = s.blocks[i];
        const int n = tiles_of(b.runs), n_pages = b.runs.pages();
        const int32_t *ids = p->host + p->off_pages + b.page_off;
        for (int c = 0; c < b.k; c++, r += kRecordInts) {
            r[RC_T0] = (int32_t)((int64_t)n * c / b.k);
            r[RC_T1] = (int32_t)((int64_t)n * (c + 1) / b.k);
            r[RC_REGION] = b.row0 < 0 ? -1 : (int32_t)(b.row0 + (int64_t)c * b.npos * G);
            r[SR_KVROWS] = (int32_t)b.kv_rows;
            r[RC_POS0] = 0;
            r[RC_NPOS] = b.npos;
            r[RC_QROW0] = b.qrow;
            r[RC_CTX] = b.pos;
            r[RC_PAGEOFF] = b.page_off;
            r[SR_A] = b.runs.a; r[SR_H] = b.runs.h; r[SR_F] = b.runs.f; r[SR_B] = b.runs.b; r[SR_C] = b.runs.c; r[SR_E] = b.runs.e;
            for (int x = 0; x < kRecordInts - RC_IDS; x++) r[RC_IDS + x] = ids[b.runs.page(std::min(r[RC_T0] * kTilePages + x, n_pages - 1))];
        }
    }
    s.n_records = (int)pieces;
    s.n_sweeps = (int)(pieces * Hkv);

    // decode items, the longest first, in whole workgroups
    s.order.resize(s.entries.size());
    std::iota(s.order.begin(), s.order.end(), 0);
    std::stable_sort(s.order.begin(), s.order.end(), [&](int x, int y) {
        return s.entries[x].runs.pages() / s.entries[x].units > s.entries[y].runs.pages() / s.entries[y].units;
    });
    const int per_wg = s.items_per_wg();
    s.n_items = (int)((units * Hkv + per_wg - 1) / per_wg * per_wg);
    s.items.assign((size_t)s.n_items * kSpanItemInts, 0);
    int32_t *d = s.items.data();
    for (const int i : s.order) {
        const SpanEntry &e = s.entries[i];
        const int64_t n = e.runs.pages();
        for (int u = 0; u < e.units; u++)
            for (int h = 0; h < Hkv; h++, d += kSpanItemInts) {
                d[SD_POS] = e.pos; d[SD_KVH] = h; d[SD_QROW] = e.qrow; d[SD_PAGEOFF] = e.page_off; d[SD_COLS] = e.cols;
                d[SD_BEGIN] = (int32_t)(n * u / e.units);
                d[SD_END] = (int32_t)(n * (u + 1) / e.units);
                d[SD_ROW] = e.row0 < 0 ? -1 : (int32_t)(e.row0 + ((int64_t)h * e.units + u) * e.cols);
                d[SD_A] = e.runs.a; d[SD_H] = e.runs.h; d[SD_F] = e.runs.f; d[SD_B] = e.runs.b; d[SD_C] = e.runs.c; d[SD_E] = e.runs.e;
            }
    }
    for (int32_t *end = s.items.data() + s.items.size(); d < end; d += kSpanItemInts) {  // padding: no pages
        d[SD_ROW] = -1;
        d[SD_COLS] = 1;
        d[SD_E] = 1;
    }
    return TC_OK;
}

SpanPart part_of(const tc_plan *p, const SpanBlock &b) { return {b.qrow, b.npos, b.k, b.row0, b.kv_rows, (int64_t)b.npos * p->G}; }
SpanPart part_of(const tc_plan *p, const SpanEntry &e) { return {e.qrow, e.cols / p->G, e.units, e.row0, (int64_t)e.units * e.cols, e.cols}; }

// Merge items: `first` and `second` say where the partial results of packed rows lie, each in the order of the rows.  Rows that are in one of them only have their results there.
void add_merges(const tc_plan *p, SpanList &s) {
    const auto by_row = [](const SpanPart &x, const SpanPart &y) { return x.qrow < y.qrow; };
    std::sort(s.first.begin(), s.first.end(), by_row);
    std::sort(s.second.begin(), s.second.end(), by_row);
    s.merge.clear();
    size_t i = 0, j = 0;
    int row = 0;
    for (;;) {
        while (i < s.first.size() && s.first[i].qrow + s.first[i].n <= row) i++;
        while (j < s.second.size() && s.second[j].qrow + s.second[j].n <= row) j++;
        const SpanPart *a = i < s.first.size() ? &s.first[i] : nullptr, *b = j < s.second.size() ? &s.second[j] : nullptr;
        if (!a && !b) break;
        row = std::max(row, std::min(a ? a->qrow : INT32_MAX, b ? b->qrow : INT32_MAX));
        if (a && a->qrow > row) a = nullptr;  // begins later
        if (b && b->qrow > row) b = nullptr;
        int end = row + kSpanMergeRows;
        for (const SpanPart *x : {a, b})
            if (x) end = std::min(end, x->qrow + x->n);
        if (!a && i < s.first.size()) end = std::min(end, s.first[i].qrow);
        if (!b && j < s.second.size()) end = std::min(end, s.second[j].qrow);
        int32_t m[kSpanItemInts] = {};
        m[SM_QROW] = row;
        m[SM_N] = end - row;
        const auto put = [&](const SpanPart *x, int at) {
            if (!x) return;
            m[at] = (int32_t)(x->row0 + (int64_t)(row - x->qrow) * p->G);
            m[at + 1] = (int32_t)x->kv_rows;
            m[at + 2] = x->count;
            m[at + 3] = (int32_t)x->step;
        };
        put(a, SM_A);
        put(b, SM_B);
        s.merge.insert(s.merge.end(), m, m + kSpanItemInts);
        row = end;
    }
    s.n_merge = (int)(s.merge.size() / kSpanItemInts);
}

void clear(SpanList &s) {
    s.ready = false;
    s.blocks.clear();
    s.entries.clear();
    s.first.clear();
    s.second.clear();
    s.merge.clear();
    s.n_records = s.n_sweeps = s.n_items = s.n_merge = 0;
    s.waves_log2 = 0;
    s.max_cols = 1;
    s.wide = false;
    s.n_rows = 0;
    s.build_ns = s.upload_ns = 0;
}

// From blocks and entries, of which the first n_first_blocks and n_first_entries are those of shared tokens, to the list on the device.
tc_status finish(tc_plan *p, SpanList &s, size_t n_first_blocks, size_t n_first_entries, void *stream, std::chrono::steady_clock::time_point t0) {
    share_out(p, s);
    if (tc_status st = lay_out(p, s)) return st;
    for (size_t i = 0; i < s.blocks.size(); i++)
        if (s.blocks[i].row0 >= 0) (i < n_first_blocks ? s.first : s.second).push_back(part_of(p, s.blocks[i]));
    for (size_t i = 0; i < s.entries.size(); i++)
        if (s.entries[i].row0 >= 0) (i < n_first_entries ? s.first : s.second).push_back(part_of(p, s.entries[i]));
    add_merges(p, s);
    s.off_records = 0;
    s.off_items = s.records.size();
    s.off_merge = s.off_items + s.items.size();
    const size_t total = std::max<size_t>(s.off_merge + s.merge.size(), 1);
    s.on_device = p->on_device;
    if (int err = begin_plan_host(&s, total)) {
        set_error(std::string("host buffer of the work list: ") + hip_error_text(err));
        return TC_ERR_DEVICE;
    }
    std::memcpy(s.host + s.off_records, s.records.data(), s.records.size() * sizeof(int32_t));
    std::memcpy(s.host + s.off_items, s.items.data(), s.items.size() * sizeof(int32_t));
    std::memcpy(s.host + s.off_merge, s.merge.data(), s.merge.size() * sizeof(int32_t));
    s.host_n = total;
    const auto t1 = std::chrono::steady_clock::now();
    s.build_ns = std::chrono::duration_cast<std::chrono::nanoseconds>(t1 - t0).count();
    if (p->on_device) {
        int device = -1, err = current_device(&device);
        if (!err && device != p->device) return fail(TC_ERR_DEVICE, "the current device is not the one the plan was made on");
        if (!err) err = upload_plan(&s, stream);
        if (err) {
            set_error(std::string("upload of the work list failed: ") + hip_error_text(err));
            return TC_ERR_DEVICE;
        }
        s.upload_ns = std::chrono::duration_cast<std::chrono::nanoseconds>(std::chrono::steady_clock::now() - t1).count();
    }
    s.ready = true;
    return TC_OK;
}

template <class F>
tc_status guarded(SpanList &s, const F &f) {
    clear(s);
    tc_status st;
    try {
        st = f();
    } catch (const std::exception &) {  // no memory for the lists
        st = fail(TC_ERR_DEVICE, "out of memory");
    }
    if (st != TC_OK) clear(s);
    return st;
}

}  // namespace

}  // namespace tc

using namespace tc;

extern "C" {

tc_status tc_plan_set_window(tc_plan *p, int32_t window, int32_t sinks, void *stream) {
    if (!p) return fail(TC_ERR_NULL, "plan is NULL");
    SpanList &s = p->window;
    const auto t0 = std::chrono::steady_clock::now();
    return guarded(s, [&]() -> tc_status {
        if (p->kvq) return fail(TC_ERR_SHAPE, "attention over a window needs a plan for pools in 16 bits");
        if (window < 1 || sinks < 0) return fail(TC_ERR_ARG, "window must be at least 1 and sinks at least 0");
        s.window = window;
        s.sinks = sinks;
        for (int q = 0; q < p->S; q++) add_sequence(p, s, q, 0);
        return finish(p, s, 0, 0, stream, t0);
    });
}

tc_status tc_plan_set_shared(tc_plan *p, int32_t num_groups, const int32_t *seq_start, const int32_t *prefix_len, void *stream) {
    if (!p) return fail(TC_ERR_NULL, "plan is NULL");
    SpanList &s = p->shared;
    const auto t0 = std::chrono::steady_clock::now();
    return guarded(s, [&]() -> tc_status {
        if (p->kvq) return fail(TC_ERR_SHAPE, "attention over shared tokens needs a plan for pools in 16 bits");
        if (num_groups < 0) return fail(TC_ERR_SPAN, "negative num_groups");
        if (num_groups > 0 && (!seq_start || !prefix_len)) return fail(TC_ERR_NULL, "seq_start or prefix_len is NULL");
        if (num_groups > 0 && (seq_start[0] != 0 || seq_start[num_groups] != p->S)) return fail(TC_ERR_SPAN, "the groups must cover the batch's sequences");
        if (num_groups == 0 && p->S > 0) return fail(TC_ERR_SPAN, "the groups must cover the batch's sequences");
        for (int g = 0; g < num_groups; g++) {
            if (seq_start[g + 1] <= seq_start[g]) return fail(TC_ERR_SPAN, "seq_start must be strictly increasing");
            const int n = prefix_len[g];
            if (n < 0 || n % kBlock) return fail(TC_ERR_SPAN, "prefix_len must be a multiple of 16");
            const int32_t *ids = p->host + p->off_pages;
            for (int q = seq_start[g]; q < seq_start[g + 1]; q++) {
                if (q >= p->S) return fail(TC_ERR_SPAN, "the groups must cover the batch's sequences");
                if (n > p->ctx_len[q]) return fail(TC_ERR_SPAN, "a sequence has fewer cached tokens than its group shares");
                if (n && std::memcmp(ids + p->page_off[q], ids + p->page_off[seq_start[g]], (size_t)(n / kBlock) * sizeof(int32_t)))
                    return fail(TC_ERR_BLOCK, "the sequences of a group do not begin with the same blocks");
            }
        }
        s.window = INT32_MAX;
        s.sinks = 0;
        // what is shared: a group's rows as one matrix, over the tokens before all of them
        for (int g = 0; g < num_groups; g++) {
            const int q0 = seq_start[g], q1 = seq_start[g + 1], pages = prefix_len[g] / kBlock;
            if (pages == 0 || q1 - q0 == 1) continue;
            const int row0 = p->q_start[q0], rows = p->q_start[q1] - row0, after = 1 << 30;
            const SpanRuns all = {pages, 0, 0, 0, 0, 0};
            if (rows * p->G <= 16) {
                s.entries.push_back({row0, rows * p->G, after, p->page_off[q0], all, true});
                continue;
            }
            const int per = kPrefillRows / p->G;
            for (int i = 0; i < rows; i += per) s.blocks.push_back({row0 + i, std::min(per, rows - i), after, p->page_off[q0], all, true});
        }
        const size_t n_blocks = s.blocks.size(), n_entries = s.entries.size();
        for (int g = 0; g < num_groups; g++) {
            const int q0 = seq_start[g], q1 = seq_start[g + 1];
            for (int q = q0; q < q1; q++) add_sequence(p, s, q, q1 - q0 > 1 ? prefix_len[g] / kBlock : 0);
        }
        return finish(p, s, n_blocks, n_entries, stream, t0);
    });
}

size_t tc_window_workspace_bytes(const tc_plan *p) { return p ? p->span_workspace_bytes(p->window) : 0; }
size_t tc_shared_workspace_bytes(const tc_plan *p) { return p ? p->span_workspace_bytes(p->shared) : 0; }

tc_status tc_plan_get_span_info(const tc_plan *p, int32_t shared, tc_span_info *info) {
    if (!p || !info) return fail(TC_ERR_NULL, "plan or info is NULL");
    const SpanList &s = shared ? p->shared : p->window;
    std::memset(info, 0, sizeof *info);
    info->ready = s.ready;
    info->num_sweeps = s.n_records;
    info->num_decode_items = s.n_items;
    info->num_merge_items = s.n_merge;
    info->waves_per_item = 1 << s.waves_log2;
    info->grid_blocks = s.ready ? s.grid_blocks() : 0;
    info->block_threads = 64 * s.waves();
    info->num_partial_rows = s.n_rows;
    info->build_ns = s.build_ns;
    info->upload_ns = s.upload_ns;
    return TC_OK;
}

tc_status tc_plan_copy_span(const tc_plan *p, int32_t shared, int32_t kind, int32_t *dst, size_t cap_items) {
    if (!p || !dst) return fail(TC_ERR_NULL, "plan or dst is NULL");
    if (kind < 0 || kind > 2) return fail(TC_ERR_ARG, "kind must be 0, 1 or 2");
    const SpanList &s = shared ? p->shared : p->window;
    if (!s.ready) return fail(TC_ERR_ARG, "the plan has no such work list");
    const size_t at[3] = {s.off_records, s.off_items, s.off_merge}, n[3] = {(size_t)s.n_records, (size_t)s.n_items, (size_t)s.n_merge};
    const size_t width = kind == 0 ? kRecordInts : kSpanItemInts, count = std::min(n[kind], cap_items);
    if (count) std::memcpy(dst, s.host + at[kind], count * width * sizeof(int32_t));
    return TC_OK;
}

}  // extern "C"
