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
constexpr int32_t kBehindAll = INT32_MAX - 1023;  // position of the rows that sweep shared tokens: behind these, and the last of a block of rows before kNoToken
constexpr int kMinSweepTiles = 4;   // a piece of a cut sweep is not shorter than this
constexpr double kAloneSmall = 0.6;  // a tile of a workgroup of four waves that has its compute unit to itself, to one of eight's
constexpr double kPieceUs = 8, kMergeUs = 8, kPartUs = 0.15;  // what a piece costs on top of its tiles: its start and end; the launch that combines pieces, and what each piece of a row adds to it
constexpr int kUncutPages = 28, kFewUncutPages = 10;   // a wave gets up to that many before an item is cut: where uncut items fill the chip, where they do not
constexpr int kShortSweepTiles = 32;
constexpr int kMinWavePages = 6;    // nor does a wave get fewer pages of a decode item that is shared out
constexpr int64_t kDecodeWaveSlots = (int64_t)kNumCu * kDecodeWgPerCu * kDecodeWaves;  // waves of decode-only workgroups that the chip holds
// Rates that the two branches are balanced with where a batch has both (one MI355X): what a sweep of 256 rows takes for a tile, and what a compute unit streams.  (A tile of long sweeps
// takes 1.71 us; the rules below were measured with 1.8.)
constexpr double kSweepTileUs = 1.8, kStreamCuBytesPerUs = 40e3, kStreamBytesPerUs = 6e6;

int tiles_of(const SpanRuns &r) { return (r.pages() + kTilePages - 1) / kTilePages; }

// Rows of one sequence (or, with `from` >= 0 and runs given by the caller, of several) in blocks that a workgroup sweeps.
void add_blocks(const tc_plan *p, SpanList &s, int seq, int from) {
    const int per = s.rows_per_block() / p->G, q = p->q_start[seq + 1] - p->q_start[seq];
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

// The sweeps in runs of equal cost, `bins` for each KV head: the blocks laid end to end, the longest first, and cut where a run is full.
void level(SpanList &s, int bins, double piece_tiles) {
    s.order.resize(s.blocks.size());
    std::iota(s.order.begin(), s.order.end(), 0);
    std::stable_sort(s.order.begin(), s.order.end(), [&](int x, int y) { return tiles_of(s.blocks[x].runs) > tiles_of(s.blocks[y].runs); });
    double left = (bins - 1) * piece_tiles;  // a cut makes one piece more
    for (const SpanBlock &b : s.blocks) left += tiles_of(b.runs) + piece_tiles;
    int run = 0;
    double room = left / bins;
    for (const int i : s.order) {
        SpanBlock &b = s.blocks[i];
        const int n = tiles_of(b.runs);
        b.k = 0;
        for (int at = 0; at < n;) {
            int take = n - at;
            const int fits = (int)(room - piece_tiles + 0.5);
            if (run + 1 < bins && fits < take) {
                if (fits < kMinSweepTiles && room < left / (bins - run) - 0.5) {  // too little for a piece: what is left is shared out over the other runs
                    run++;
                    room = left / (bins - run);
                    continue;
                }
                const int cut = std::max(fits, kMinSweepTiles);
                if (take - cut >= kMinSweepTiles) take = cut;
            }
            s.pieces.push_back({i, at, at + take, b.k++, run});
            at += take;
            room -= take + piece_tiles;
            left -= take + piece_tiles;
            if (run + 1 < bins && room < kMinSweepTiles) {
                run++;
                room = left / (bins - run);
            }
        }
    }
}

// The pieces of the sweeps and the waves of the decode items.
void share_out(const tc_plan *p, SpanList &s) {
    const int64_t Hkv = p->Hkv;
    int64_t tiles = 0, longest = 0, pages = 0;
    for (const SpanBlock &b : s.blocks) {
        tiles += tiles_of(b.runs);
        longest = std::max<int64_t>(longest, tiles_of(b.runs));
    }
    for (const SpanEntry &e : s.entries) pages += e.runs.pages();
    const bool sweeps = !s.blocks.empty();
    const int waves = s.blocks.empty() ? kDecodeWaves : s.sweep_waves;
    const int64_t wg_slots = sweeps ? (int64_t)kNumCu * (s.sweep_waves == kMixedWaves ? 1 : small_wg_per_cu(p->D)) : kNumCu * kDecodeWgPerCu;
    const double tile_us = kSweepTileUs * p->D / 128 * s.sweep_waves / kMixedWaves;  // of a workgroup's share of its compute unit
    const double sweep_us = ((double)tiles * tile_us + (double)s.blocks.size() * kPieceUs) * Hkv;
    const double bytes = (double)pages * Hkv * kBlock * p->token_bytes(), stream_us = bytes / kStreamCuBytesPerUs;
    const double share = sweep_us / std::max(1e-9, sweep_us + stream_us);  // of the compute units that sweep
    if (sweeps) {
        const int64_t whole = (int64_t)s.blocks.size() * Hkv;
        const int64_t target = std::max<int64_t>(Hkv, (int64_t)((double)kNumCu * (pages > 0 ? share : 1.0)));  // compute units that sweep at a time
        // Fewer blocks than units: whole, or in level runs, which pay a start and an end for each piece and a launch that combines them; one run to a unit, or as many as it holds where the
        // tiles are many.  Not beside a stream that takes longer than the longest sweep.  (us, one / as many as fit, head_dim 64: 97 tokens behind 4769, 32/8 heads, 20 / 28; 19 decodes
        // behind 15264, 32/8, 20 / 25; 234 tokens and 17 decodes behind 9280, 32/32, 88 / 47; 249 decodes behind 6704, 64/8, 66 / 54.)
        const double alone_us = kSweepTileUs * p->D / 128 * (s.sweep_waves == kMixedWaves ? 1.0 : kAloneSmall), all_us = bytes / kStreamBytesPerUs;
        double best = 0.95 * std::max((double)longest * alone_us + kPieceUs, all_us);
        double piece_tiles = 0;
        int64_t bins = 0;
        for (int64_t r = 1, per_cu = wg_slots / kNumCu; whole < target && r <= per_cu; r++) {
            const int64_t n = std::max<int64_t>(1, std::min<int64_t>(target * r / Hkv, tiles / kMinSweepTiles));
            const double run_us = std::max(alone_us, tile_us * std::max(1.0, (double)(n * Hkv) / kNumCu));  // a tile of a run beside the others of its unit
            const double parts = (double)longest * (double)n / (double)tiles;
            const double t = std::max(((double)tiles * run_us + (double)((int64_t)s.blocks.size() + n - 1) * kPieceUs) / (double)n + kMergeUs + kPartUs * parts, all_us);
            if (t < best) best = t, bins = n, piece_tiles = kPieceUs / run_us;
        }
        if (bins > 0) level(s, (int)bins, piece_tiles);
    }
    if (s.pieces.empty())
        for (size_t i = 0; i < s.blocks.size(); i++) s.pieces.push_back({(int32_t)i, 0, tiles_of(s.blocks[i].runs), 0, (int32_t)i});

    // Pages of a wave: as many as keep all waves that the chip holds busy, but no fewer than are worth a wave.
    // (Beside sweeps half as many: finer units for the units that sweeps leave free.)
    const int64_t slots = wg_slots * waves * (sweeps ? 2 : 1), least = kMinWavePages;
    const int64_t per_wave = std::min<int64_t>(kMaxSplitPages, std::max<int64_t>(least, (pages * Hkv + slots - 1) / slots));
    s.waves_log2 = 0;
    if (!s.entries.empty()) {
        const int64_t mean = (pages + (int64_t)s.entries.size() - 1) / (int64_t)s.entries.size();
        while ((1 << s.waves_log2) < waves && ((int64_t)per_wave << s.waves_log2) < mean) s.waves_log2++;
    }
    s.wide = !sweeps && (pages * Hkv + per_wave - 1) / per_wave <= (int64_t)kNumCu * 2 * kDecodeWaves;
    // A sequence is cut into several items only where that saves more pages a wave than the launch that combines them costs.
    const int64_t most = std::min<int64_t>((int64_t)kMaxSplitPages << s.waves_log2, std::max<int64_t>(per_wave + per_wave / 2, (int64_t)s.entries.size() * Hkv >= kNumCu ? kUncutPages : kFewUncutPages) << s.waves_log2);
    int64_t n_items = 0;
    for (SpanEntry &e : s.entries) {
        const int64_t n = e.runs.pages(), each = e.partial ? std::min<int64_t>(per_wave + per_wave / 2, kMaxSplitPages) << s.waves_log2 : n <= most ? most : per_wave << s.waves_log2;
        e.units = (int32_t)((n + each - 1) / each);
        n_items += e.units * Hkv;
    }
    // More workgroups than the chip holds: the launch begins with a mix of both kinds.
    s.n_first = s.n_early = 0;
    int64_t n_sweeps = 0;
    for (size_t i = 0; i < s.pieces.size(); i++) n_sweeps += (i == 0 || s.pieces[i].run != s.pieces[i - 1].run) * Hkv;
    const int64_t units = (n_items + (waves >> s.waves_log2) - 1) / (waves >> s.waves_log2);
    if (sweeps && n_items > 0 && n_sweeps + units > wg_slots) {
        s.n_first = (int)std::min<int64_t>(n_sweeps, std::max<int64_t>(1, (int64_t)((double)wg_slots * share / Hkv + 0.5)) * Hkv);
        s.n_early = (int)(std::min<int64_t>(units, std::max<int64_t>(wg_slots - s.n_first, 0)) / Hkv * Hkv);
    }
}

// Tiles of the longest sequence that a sweep may cover.
int64_t longest_chunk(const tc_plan *p) {
    int64_t n = 0;
    for (int q = 0; q < p->S; q++) n = std::max<int64_t>(n, p->ctx_len[q] + (p->q_start[q + 1] - p->q_start[q]));
    return (n + kPrefillTileTokens - 1) / kPrefillTileTokens;
}

// Workgroups of four waves, several to a compute unit, where sweeps are short: one's start and end run beside another's tiles, or a sweep beside decodes.  (us, four waves / eight.
// Windows: 64/8 heads, head_dim 128, 8192 tokens, of 512 213 / 235, 1024 328 / 325, 2048 556 / 538, 5000 1213 / 1144; 32/8, 2000 with 60 decodes, 512 47 / 53, 2048 112 / 132, 5000
// 222 / 236; 500 with 60 decodes, 512 28 / 42, 2048 81 / 94, 5000 135 / 125; head_dim 64, 64/8, 8192, 512 109 / 137, 2048 314 / 338, 5000 701 / 697.  Shared tokens:
// 300 decodes behind 1024, 32/8, 76 / 83, 64 behind 2048 26 / 26, 128 behind 8192 65 / 51; head_dim 64, 16/2, 128 behind 8192 22 / 25, 100 behind 16384 24 / 28.)
int choose_sweep_waves(int64_t tiles, int64_t short_tiles) { return tiles <= short_tiles ? kSmallWaves : kMixedWaves; }

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

    // Pieces in the order of their runs, whole blocks the longest first; the records of the runs' first pieces come first, those of the others behind them.
    if (pieces == (int64_t)s.blocks.size())
        std::stable_sort(s.pieces.begin(), s.pieces.end(), [](const SpanPiece &x, const SpanPiece &y) { return x.t1 - x.t0 > y.t1 - y.t0; });
    int n_runs = 0;
    for (size_t i = 0; i < s.pieces.size(); i++) n_runs += i == 0 || s.pieces[i].run != s.pieces[i - 1].run;
    s.records.assign((size_t)pieces * kRecordInts, 0);
    int32_t first = 0, next = n_runs, *before = nullptr;
    for (size_t i = 0; i < s.pieces.size(); i++) {
        const SpanPiece &x = s.pieces[i];
        const SpanBlock &b = s.blocks[x.block];
        const bool begins = i == 0 || x.run != s.pieces[i - 1].run;
        const int32_t index = begins ? first++ : next++;
        if (!begins) before[SR_NEXT] = index;
        int32_t *r = s.records.data() + (size_t)index * kRecordInts;
        before = r;
        const int32_t *ids = p->host + p->off_pages + b.page_off;
        const int n_pages = b.runs.pages();
        r[RC_T0] = x.t0;
        r[RC_T1] = x.t1;
        r[RC_REGION] = b.row0 < 0 ? -1 : (int32_t)(b.row0 + (int64_t)x.c * b.npos * G);
        r[SR_KVROWS] = (int32_t)b.kv_rows;
        r[SR_NEXT] = -1;
        r[RC_POS0] = 0;
        r[RC_NPOS] = b.npos;
        r[RC_QROW0] = b.qrow;
        r[RC_CTX] = b.pos;
        r[RC_PAGEOFF] = b.page_off;
        r[SR_A] = b.runs.a; r[SR_H] = b.runs.h; r[SR_F] = b.runs.f; r[SR_B] = b.runs.b; r[SR_C] = b.runs.c; r[SR_E] = b.runs.e;
        for (int at = 0; at < kRecordInts - RC_IDS; at++) r[RC_IDS + at] = ids[b.runs.page(std::min(x.t0 * kTilePages + at, n_pages - 1))];
    }
    s.n_records = (int)pieces;
    s.n_sweeps = n_runs * Hkv;

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
        s.merge_rows = std::max(s.merge_rows, end - row);
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

// Decodes alone, over a window or in groups that share nothing, a workgroup to an item, and not too many of them: the last workgroup of a sequence and KV head to leave a partial result
// combines them.  (Where tokens are shared the rows of a group would be combined by one workgroup, one after the other: 4 decodes behind 2048 shared tokens, 32/8 heads, 15 us, with a
// second launch 11.)
void fuse(const tc_plan *p, SpanList &s) {
    s.fused = s.blocks.empty() && s.first.empty() && s.n_merge > 0 && s.items_per_wg() == 1 && (int64_t)s.n_merge * p->Hkv <= kCounterInts && s.n_rows * p->D * 4 < (int64_t)1 << 31;
    if (!s.fused) return;
    s.counter_stride = kCounterLine;
    while ((int64_t)s.n_merge * p->Hkv * s.counter_stride > kCounterInts) s.counter_stride /= 2;
    s.order.assign((size_t)p->T, -1);  // the merge item of each row
    for (int m = 0; m < s.n_merge; m++) s.order[s.merge[(size_t)m * kSpanItemInts + SM_QROW]] = m;
    for (size_t i = 0; i < s.items.size(); i += kSpanItemInts) {
        int32_t *d = s.items.data() + i;
        if (d[SD_ROW] < 0) continue;
        d[SD_MERGE] = s.order[d[SD_QROW]];
        d[SD_PARTS] = s.merge[(size_t)d[SD_MERGE] * kSpanItemInts + SM_NB];
    }
}

void clear(SpanList &s) {
    s.ready = false;
    s.blocks.clear();
    s.entries.clear();
    s.pieces.clear();
    s.first.clear();
    s.second.clear();
    s.merge.clear();
    s.n_records = s.n_sweeps = s.n_items = s.n_merge = 0;
    s.waves_log2 = 0;
    s.max_cols = s.merge_rows = 1;
    s.wide = s.fused = false;
    s.n_first = s.n_early = 0;
    s.sweep_waves = kMixedWaves;
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
    fuse(p, s);
    s.off_records = 0;
    s.off_items = s.records.size();
    s.off_merge = s.off_items + s.items.size();
    s.off_counters = (s.off_merge + s.merge.size() + kCounterLine - 1) / kCounterLine * kCounterLine;
    const size_t n_counters = s.fused ? (size_t)s.n_merge * p->Hkv * s.counter_stride : 0, total = std::max<size_t>(s.off_counters + n_counters, 1);
    s.on_device = p->on_device;
    if (int err = begin_plan_host(&s, total)) {
        set_error(std::string("host buffer of the work list: ") + hip_error_text(err));
        return TC_ERR_DEVICE;
    }
    std::memcpy(s.host + s.off_records, s.records.data(), s.records.size() * sizeof(int32_t));
    std::memcpy(s.host + s.off_items, s.items.data(), s.items.size() * sizeof(int32_t));
    std::memcpy(s.host + s.off_merge, s.merge.data(), s.merge.size() * sizeof(int32_t));
    std::memset(s.host + s.off_counters, 0, n_counters * sizeof(int32_t));
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
        // (the tiles of a block of 256 rows in the middle of a long sequence)
        s.sweep_waves = choose_sweep_waves(std::min<int64_t>(((int64_t)window + sinks) / kPrefillTileTokens + 2, longest_chunk(p)), (p->D == 64 || p->n_decode_seqs > 0 ? 2 : 1) * kShortSweepTiles);
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
        s.sweep_waves = choose_sweep_waves(longest_chunk(p), p->D == 64 ? INT64_MAX : kShortSweepTiles);
        // What is shared: the rows of a group's sequences as one matrix, over the tokens before all of them.  A chunk that fills a block of rows by itself has its own sweep over
        // everything, which reads what is shared once for the block as well and leaves nothing to combine; the sequences between such chunks are taken together.
        const auto alone = [&](int q) { return (int64_t)(p->q_start[q + 1] - p->q_start[q]) * p->G >= kPrefillRows; };
        const auto together = [&](int q, int q1) {  // end of the run of sequences from q on that are taken together
            while (q < q1 && !alone(q)) q++;
            return q;
        };
        for (int g = 0; g < num_groups; g++) {
            const int q1 = seq_start[g + 1], pages = prefix_len[g] / kBlock;
            for (int q = seq_start[g], end; q < q1 && pages > 0; q = std::max(end, q + 1)) {
                end = together(q, q1);
                if (end - q < 2) continue;
                if (prefix_len[g] > kBehindAll) return fail(TC_ERR_SPAN, "more than 2^31 - 1024 shared tokens");
                const int row0 = p->q_start[q], rows = p->q_start[end] - row0;
                const SpanRuns all = {pages, 0, 0, 0, 0, 0};
                if (rows <= 16 / p->G) {
                    s.entries.push_back({row0, rows * p->G, kBehindAll, p->page_off[q], all, true});
                    continue;
                }
                const int per = s.rows_per_block() / p->G;
                for (int i = 0; i < rows; i += per) s.blocks.push_back({row0 + i, std::min(per, rows - i), kBehindAll, p->page_off[q], all, true});
            }
        }
        const size_t n_blocks = s.blocks.size(), n_entries = s.entries.size();
        for (int g = 0; g < num_groups; g++) {
            const int q1 = seq_start[g + 1];
            for (int q = seq_start[g]; q < q1;) {
                const int end = std::max(together(q, q1), q + 1);
                const int from = end - q < 2 ? 0 : prefix_len[g] / kBlock;
                for (; q < end; q++) add_sequence(p, s, q, from);
            }
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
    info->num_sweep_workgroups = s.n_sweeps;
    info->num_decode_items = s.n_items;
    info->num_merge_items = s.n_merge;
    info->merge_launch = s.n_merge > 0 && !s.fused;
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
