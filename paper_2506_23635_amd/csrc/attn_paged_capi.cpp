// attn_paged_capi.cpp -- the C-ABI of the paged cache (include/attn.h):
// configuration checks, the carve-up of the caller's cache and workspace, a
// batch's checks and its division into workgroups' shares, and the launches.
// Nothing here allocates device memory.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <functional>
#include <new>
#include <queue>
#include <string>
#include <utility>
#include <vector>

#include "attn_paged.h"

using paged::Item;
using paged::Merge;

namespace {

constexpr size_t kAlign = 256;
constexpr int kStages = 4;             // batches on their way to the device at once
using paged::kXcds;
using paged::kFewRuns;
// Dividing positions makes at most twice as many shares (and partial sums) of tile()
constexpr int64_t kTileItems = 768;
constexpr int kMostRanges = 16;        // of one row block (the merge's waves take a row of 16 slots)
constexpr int kFewStep = 4 * paged::kTile;   // positions of a workgroup's step of few()
constexpr double kStreamRate = 6.3e6;  // bytes/us that few() reads where every CU has its share
constexpr int kGraphGrid = 512;        // workgroups that a captured launch has at least of a kind,
constexpr int kGraphMerge = 16;        // and entries of its merge at once

size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

struct Layout {
    size_t data_bytes, scale_bytes, layer_bytes, cache_bytes;   // K or V of a layer; its scales
    size_t hdr, freq, tok, pages, few, tile[2], merge[2], table, few_part, tile_part, ws_bytes;
    size_t max_few, max_tile[2], max_merge[2], few_slots, tile_slots;
    int shift;
};

const char* check_config(const attn_paged_config* c)
{
    if (!c) return "config is NULL";
    if (c->head_dim != 64 && c->head_dim != 128) return "head_dim must be 64 or 128";
    if (c->n_heads < 1 || c->n_kv_heads < 1 || c->n_heads % c->n_kv_heads) return "n_kv_heads must divide n_heads";
    if (c->n_heads / c->n_kv_heads > paged::kFewRows) return "at most 16 query heads per key/value head";
    if ((int64_t)c->n_heads * c->head_dim > 65536) return "n_heads * head_dim too large";
    if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)))
        return "page_size must be 16, 32, 64, 128 or 256";
    if (c->n_pages < 1 || c->n_pages > (1 << 24)) return "n_pages must be in [1, 2^24]";
    if (c->n_layers < 1 || c->n_layers > 1024) return "n_layers must be in [1, 1024]";
    if (c->max_seqs < 1 || c->max_seqs > 4096) return "max_seqs must be in [1, 4096]";
    if (c->max_tokens < 1 || c->max_tokens > 32768) return "max_tokens must be in [1, 32768]";
    if (c->max_blocks < 1 || c->max_blocks > 65536) return "max_blocks must be in [1, 65536]";
    if ((int64_t)c->max_blocks * c->page_size > (1 << 24)) return "max_blocks * page_size must be at most 2^24";
    if ((int64_t)c->max_seqs * c->max_blocks > (1 << 26)) return "max_seqs * max_blocks must be at most 2^26";
    if (!(c->rope_theta > 1.0f) || !std::isfinite(c->rope_theta)) return "rope_theta must be > 1";
    if (c->flags & ~ATTN_PAGED_E4M3) return "flags must be 0 or ATTN_PAGED_E4M3";
    return nullptr;
}

Layout make_layout(const attn_paged_config* c)
{
    Layout L{};
    const size_t G = c->n_kv_heads, hd = c->head_dim, H = c->n_heads, group = H / G;
    const bool e4m3 = c->flags & ATTN_PAGED_E4M3;
    for (L.shift = 4; (1 << L.shift) < c->page_size; ++L.shift) {}
    L.data_bytes = (size_t)c->n_pages * G * c->page_size * hd * (e4m3 ? 1 : 2);
    L.scale_bytes = e4m3 ? align_up((size_t)c->n_pages * G * 4, kAlign) : 0;
    L.layer_bytes = 2 * L.data_bytes + 2 * L.scale_bytes;
    L.cache_bytes = L.layer_bytes * c->n_layers;
    // Shares: every sequence and key/value head has one, every row block of
    // tile(), and divided positions add one for each end of a run of few(), and
    // of tile() at most twice the division's aim (a range is at least half as
    // long as the common length).
    const size_t S = c->max_seqs, T = c->max_tokens, rows = T * group;
    const size_t few_seqs = std::min(S, T), tile_seqs = std::min(S, rows / (paged::kFewRows + 1) + 1);
    // (at least kGraphGrid, and eight more, as a launch's workgroups are a multiple of eight)
    L.max_few = few_seqs * G + kFewRuns + kXcds;
    // (every end of a run makes a share, and its neighbour, two of several; no more than steps)
    const size_t few_steps = few_seqs * G * (((size_t)c->max_blocks * c->page_size + kFewStep - 1) / kFewStep);
    L.few_slots = std::min<size_t>(2 * kFewRuns, few_steps);
    const bool tiles = rows > (size_t)paged::kFewRows;
    for (int k = 0; k < 2; ++k)
        L.max_tile[k] = tiles ? (rows / (128 >> k) + tile_seqs) * G + 2 * kTileItems + kXcds : 0;
    // (a row block has at most kMostRanges ranges, and no more than steps; blocks
    // of 64 rows are the most there are)
    const size_t tile_steps = ((size_t)c->max_blocks * c->page_size + paged::kStep - 1) / paged::kStep;
    const size_t most = std::min<size_t>(kMostRanges, tile_steps);
    L.tile_slots = tiles && most > 1 ? std::min<size_t>(2 * kTileItems, (rows / 64 + tile_seqs) * G * most) : 0;
    L.max_merge[0] = std::max<size_t>(kFewRuns, kGraphMerge);
    L.max_merge[1] = tiles ? kTileItems : 0;
    size_t off = 0;
    auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes, kAlign); return o; };
    L.hdr = take(sizeof(paged::Header));
    L.freq = take(hd / 2 * 8);
    L.tok = take(T * sizeof(paged::Token) + 16);
    L.pages = take(T * sizeof(paged::PageWork));
    L.few = take(L.max_few * sizeof(Item));
    L.tile[0] = take(L.max_tile[0] * sizeof(Item));
    L.tile[1] = take(L.max_tile[1] * sizeof(Item));
    L.merge[0] = take(L.max_merge[0] * sizeof(Merge));
    L.merge[1] = take(L.max_merge[1] * sizeof(Merge));
    L.table = take(S * c->max_blocks * 4 + 16);
    L.few_part = take(L.few_slots * paged::kFewRows * (hd + paged::kPartPad) * 4);
    L.tile_part = take(L.tile_slots * 128 * (hd + paged::kPartPad) * 4);
    L.ws_bytes = off;
    return L;
}

thread_local std::string g_init_error;

struct Stage {
    uint8_t* mem = nullptr;            // pinned host memory
    size_t bytes = 0;
    hipEvent_t done = nullptr;
    bool busy = false;
};

// A batch as the host keeps it.
struct Batch {
    std::vector<paged::Token> tok;
    std::vector<paged::PageWork> pages;
    std::vector<Item> few, tile[2];
    std::vector<Merge> merge, tile_merge;   // of few(), of tile()
    std::vector<int32_t> table;
    bool unplaced = false;                 // a new token has no page
    int n_runs = 0;                        // of few()
    int slots[2] = {0, 0};                 // most of one entry of few()'s, of tile()'s
    int all_slots[2] = {0, 0};
};

}  // namespace

struct attn_paged_ctx {
    attn_paged_config cfg;
    Layout L;
    uint8_t *cache, *ws;
    std::vector<double> freq;
    std::vector<int32_t> written;      // per page: the call that last had it written, for set_batch
    int32_t call;
    bool set, unplaced;
    bool handed;                       // the device has, or may have, a batch with tokens
    int32_t T, n_pages, n_few, n_tile[2], n_merge[2];
    int slots[2];                      // the most of one merge entry
    Stage stage[kStages];
    int next_stage;
    std::string err;
};

namespace {

moe_status fail(attn_paged_ctx* ctx, moe_status s, const char* msg)
{
    try {
        (ctx ? ctx->err : g_init_error) = msg;
    } catch (...) {
    }
    return s;
}

moe_status hip_fail(attn_paged_ctx* ctx, hipError_t e, const char* what)
{
    try {
        ctx->err = std::string(what) + ": " + hipGetErrorString(e);
    } catch (...) {
    }
    return MOE_E_HIP;
}

bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }

bool overlap(const void* a, uint64_t a_bytes, const void* b, uint64_t b_bytes)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return x < y ? y - x < a_bytes : x - y < b_bytes;
}

// of the batch's queries, or of their results
uint64_t q_bytes(const attn_paged_ctx* c) { return (uint64_t)c->T * c->cfg.n_heads * c->cfg.head_dim * 2; }

// Appends the shares of `it` that end after the given steps (the last: all of them).
void add_ranges(std::vector<Item>& out, Item it, const std::vector<int>& cuts, int step, int& slot)
{
    const int begin = it.begin, end = it.end;
    const bool several = cuts.size() > 1;
    int from = 0;
    for (int to : cuts) {
        it.begin = begin + from * step;
        it.end = (int)std::min<int64_t>(end, begin + (int64_t)to * step);
        it.slot = several ? slot++ : -1;
        out.push_back(it);
        from = to;
    }
}

// n ranges of `steps` steps that differ by one at most
void even_cuts(int64_t steps, int64_t n, std::vector<int>& cuts)
{
    cuts.clear();
    for (int64_t i = 1; i <= n; ++i) cuts.push_back((int)(steps * i / n));
}

// A row block of tile(): the steps of 64 positions that it needs, and the
// number of ranges that they are divided into.
struct Block {
    int steps, rows, ranges;
};

// How long workgroups take together, their times alone on a CU given longest
// first: handed out in that order, one to each CU, then a second, then to
// whichever has one done; two on a CU each take `slow` times as long.
double play(const std::vector<double>& times, int cus, double slow)
{
    struct Cu {
        double left[2], at;
        int n;
        unsigned version;                                // of its event in the queue
    };
    typedef std::pair<double, std::pair<int, unsigned>> Event;
    std::vector<Cu> cu(cus, Cu{});
    std::priority_queue<Event, std::vector<Event>, std::greater<Event>> events;
    size_t next = 0;
    double end = 0.0;
    auto fill = [&](Cu& c) {
        if (next < times.size()) c.left[c.n++] = times[next++];
    };
    auto schedule = [&](int x) {
        Cu& c = cu[x];
        ++c.version;
        if (c.n == 1) events.push({c.at + c.left[0], {x, c.version}});
        if (c.n == 2) events.push({c.at + std::min(c.left[0], c.left[1]) * slow, {x, c.version}});
    };
    for (int k = 0; k < 2; ++k)
        for (Cu& c : cu) fill(c);
    for (int x = 0; x < cus; ++x) schedule(x);
    while (!events.empty()) {
        const Event e = events.top();
        events.pop();
        Cu& c = cu[e.second.first];
        if (e.second.second != c.version) continue;
        const double done = c.n == 2 ? std::min(c.left[0], c.left[1]) : c.left[0];
        c.at = end = e.first;
        int n = 0;
        for (int k = 0; k < c.n; ++k)
            if (c.left[k] > done) c.left[n++] = c.left[k] - done;
        for (int gone = c.n - n; c.n = n, gone > 0; --gone, n = c.n) fill(c);
        schedule(e.second.first);
    }
    return end;
}

// Divides the row blocks' positions into ranges: the longest block's into 1 ..
// kMostRanges, and every block then has ranges of about that length; by the
// least estimated time, which it returns.  The workgroups are played through
// for one key/value head and its share of the CUs.  Measured at head_dim 128,
// with weights of one bf16 term: a step of 128 rows 1.25 us, where a CU has two
// workgroups 2.2, of 64 rows 0.9 and 1.35 (with the two terms that tile() takes
// 1.55, 2.65, 1.0 and 1.55; but planned with these, 500-token prompts took 20.5
// -> 17.6 us, 16 sequences of 8 tokens 41 -> 46, 20 tokens and a piece 50.8 ->
// 54.1, and the other 22 batches the same); 1.5 and 2.5 steps more per share, and one for the masks of a block's
// last; the partial sums written and read at about 9 TB/s, the merge 5 us.  (512
// tokens after 8000 positions, bf16: 1 range 192 us, 2 165, 3 208, 4 181, 5 168.)
// Beside few()'s shares, which take few_us by themselves, the longest has a
// neighbour for as long, and the work adds up (24 single tokens and two pieces:
// 1, 2, 3, 4 ranges 73.7, 62.1, 66.4, 66.3 us; the pieces alone 59, 46, 45, 44).
// The factors: 0.66 a step's time at head_dim 64 to 128's; 0.97 keeps the fewer
// ranges where the estimates are as good as equal.
double divide_blocks(std::vector<Block>& blocks, int G, int head_dim, bool wide, double few_us)
{
    constexpr int kCus = 256;
    const double step_us = (wide ? 1.25 : 0.9) * (head_dim == 128 ? 1.0 : 0.66), slow = wide ? 1.76 : 1.5, start = wide ? 1.5 : 2.5;
    const int cus = std::max(1, kCus / G);
    int longest = 0;
    double all = 0.0;
    for (Block& b : blocks) {
        b.ranges = 1;
        longest = std::max(longest, b.steps);
        all += (b.steps + start + 1.0) * step_us;
    }
    if (blocks.size() >= 8 * (size_t)cus) return all * slow / (2 * cus);   // enough without
    std::vector<double> times;
    double best_us = 0.0;
    int best_len = longest;
    for (int n = 1; n <= kMostRanges && n <= longest; n += n < 6 ? 1 : 2) {
        const int len = (longest + n - 1) / n;
        int64_t slots = 0, rows = 0;
        times.clear();
        for (const Block& b : blocks) {
            const int ranges = (b.steps + len - 1) / len;
            for (int64_t i = 0; i < ranges; ++i)
                times.push_back(((b.steps * (i + 1) / ranges - b.steps * i / ranges) + start + (i + 1 < ranges ? 0.0 : 1.0)) * step_us);
            if (ranges > 1) {
                slots += ranges;
                rows += (int64_t)ranges * b.rows;
            }
        }
        if (slots * G > 2 * kTileItems || (n > 1 && times.size() > 4 * (size_t)cus)) break;
        std::sort(times.begin(), times.end(), std::greater<double>());
        double us = play(times, cus, slow);
        if (few_us > 0.0) {
            double work = 0.0;
            for (double t : times) work += t;
            const double beside = std::min(times[0] * slow, times[0] + few_us);
            us = std::max({us, beside, few_us + work * slow / (2 * cus)});
        }
        if (slots) us += 5.0 + (double)rows * G * (head_dim + paged::kPartPad) * 4 * 2 / 9e6;
        if (n == 1 || us < 0.97 * best_us) {
            best_us = us;
            best_len = len;
        }
    }
    for (Block& b : blocks) b.ranges = (b.steps + best_len - 1) / best_len;
    return best_us;
}

// Longest shares first: the workgroups are handed out in order.
bool longer(const Item& x, const Item& y) { return x.end - x.begin > y.end - y.begin; }

// Divides the shares of few(), given as whole sequences (one per sequence and
// key/value head), into the runs of kFewRuns workgroups, equal in steps: a CU
// holds about 64 KB of loads in flight, whether of one workgroup or of two, so
// that the positions of every CU have to be as many (320 equal sequences and
// heads, one or two a CU, stream 4.7 TB/s; 256 and 512 6.3).  A run takes the
// sequences one after another, long and short ones in turn, each start counted
// as kStart steps; a sequence that runs share is added up by the merge.
// Sequences stay whole, a workgroup each, where that is estimated to take no
// longer: a CU does a step in step_us at least, or all of them stream at
// kStreamRate; divided, a merge comes after them (kMergeUs).  1.28 is what two
// shares on a CU cost beside the mean and a quarter of the longest, fitted to
// the batches below; 0.9 divides only where the estimates differ.  (bf16, from memory: one token after 256,
// 511, 1023 and 2047 positions whole 7.9, 10.9, 17.5 and 31 us, divided 11.0,
// 10.2, 10.4 and 11.0; 32 sequences of 300 to 1000 whole 21.8, 25.9 in equal
// ranges; 64 of 300 to 3000 whole 87, in equal ranges of each sequence 81, in
// runs 78; 8 of 3000 to 8000 45.3 and 42.2.)
void divide_few(std::vector<Item>& whole, double step_bytes, Batch& b, int& slot)
{
    constexpr double kStart = 0.5, kCus = 256.0, kMergeUs = 4.5;
    const double step_us = std::max(0.65, 1.68 * step_bytes / 65536);
    auto steps = [](const Item& it) { return (it.end + kFewStep - 1) / kFewStep; };
    std::stable_sort(whole.begin(), whole.end(), longer);
    int64_t total = 0;
    for (const Item& it : whole) total += steps(it);
    b.n_runs = (int)whole.size();
    b.few = whole;
    if (whole.empty() || whole.size() >= 4 * kFewRuns) return;   // (so many even out)
    const int longest = steps(whole[0]);
    const double stream_us = total * step_bytes / kStreamRate, mean = total / kCus;
    const double busiest = whole.size() <= kCus ? longest : std::max((double)longest, 1.28 * (mean + longest / 4.0));
    const double whole_us = std::max(stream_us, step_us * busiest);
    const double divided_us = std::max(stream_us, step_us * std::ceil(mean)) + kMergeUs;
    if (whole_us < 0.9 * divided_us) return;
    std::vector<int> first;                              // of each run
    for (double room_all = std::max(kStart + 1.0, (total + kStart * (whole.size() + kFewRuns)) / kFewRuns);; room_all *= 1.02) {
        b.few.clear();
        b.merge.clear();
        first.assign(1, 0);
        slot = b.slots[0] = 0;
        double room = room_all;
        for (size_t i = 0; i < whole.size(); ++i) {
            Item it = whole[i % 2 ? whole.size() - 1 - i / 2 : i / 2];
            const int end = it.end, n = steps(it);
            const size_t at = b.few.size();
            for (int from = 0; from < n;) {
                int k = n - from;
                if (k + kStart > room + std::min(1.0, room_all / 8)) {   // (rather a little longer than one more start)
                    k = (int)(room - kStart);
                    if (k < 1 || (k < 2 && room < room_all)) {
                        first.push_back((int)b.few.size());
                        room = room_all;
                        continue;
                    }
                }
                it.begin = from * kFewStep;
                it.end = std::min(end, (from + k) * kFewStep);
                b.few.push_back(it);
                from += k;
                room -= k + kStart;
            }
            const int pieces = (int)(b.few.size() - at);
            if (pieces == 1) continue;
            b.merge.push_back(Merge{it.tok0, 0, it.rows, it.kvh, slot, pieces, {}});
            b.slots[0] = std::max(b.slots[0], pieces);
            for (int k = 0; k < pieces; ++k) b.few[at + k].slot = slot++;
        }
        if (first.size() <= (size_t)kFewRuns) break;
    }
    // the list: the runs' first shares, then the others
    std::vector<Item> shares(b.few.size());
    const int runs = (int)first.size();
    int more = runs;
    first.push_back((int)b.few.size());
    for (int r = 0; r < runs; ++r) {
        int to = r;
        for (int i = first[r]; i < first[r + 1]; ++i) {
            shares[to] = b.few[i];
            const int next = i + 1 < first[r + 1] ? more++ : -1;
            shares[to].next = next;
            to = next;
        }
    }
    b.few = std::move(shares);
    b.n_runs = runs;
}

// One list for eight XCDs, workgroup b going to XCD b % 8: the shares in
// order (those of one sequence and key/value head together, so that an L2
// reads its keys and values once) cut into eight runs of about equal work,
// each run's longest first, and the runs interleaved.
void by_xcd(std::vector<Item>& v)
{
    if (v.size() <= 1) return;
    int64_t total = 0;
    auto cost = [](const Item& it) { return (int64_t)(it.end - it.begin) + 2 * paged::kStep; };
    for (const Item& it : v) total += cost(it);
    std::vector<Item> run[kXcds];
    int64_t at = 0;
    for (const Item& it : v) {
        const int64_t mid = at + cost(it) / 2;
        run[std::min<int64_t>(kXcds - 1, mid * kXcds / total)].push_back(it);
        at += cost(it);
    }
    for (auto& r : run) std::stable_sort(r.begin(), r.end(), longer);
    // a run that is used up goes on with the last of the longest one left
    std::vector<Item> out;
    out.reserve(v.size());
    size_t next[kXcds] = {};
    while (out.size() < v.size()) {
        auto left = [&](int x) { return run[x].size() - next[x]; };
        const int x = (int)(out.size() % kXcds);
        if (left(x) > 0) {
            out.push_back(run[x][next[x]++]);
            continue;
        }
        int y = 0;
        for (int k = 1; k < kXcds; ++k)
            if (left(k) > left(y)) y = k;
        out.push_back(run[y].back());
        run[y].pop_back();
    }
    v = std::move(out);
}

void divide(const attn_paged_config& c, const Layout& L, const int32_t* n_new, const int32_t* pos0, int n_seqs,
            const std::vector<uint8_t>& holes, Batch& b)
{
    const int G = c.n_kv_heads, group = c.n_heads / G;
    auto blocks_of = [&](int s) { return (int)(((int64_t)pos0[s] + n_new[s] + c.page_size - 1) >> L.shift); };
    // Row blocks of one key/value head: of 128 rows (64 where a sequence has no
    // more), or of 64 all of them where that is estimated to be quicker: twice as
    // many shares, and shorter steps, but a third more work.  (Prompts of 300, 1000
    // and 2048 tokens: 15.4, 36.9 and 84 us in blocks of 128, 12.9, 34.0 and 98 of
    // 64; four of 200 to 400 22.0 and 25.9.)  Not beside few()'s shares, which
    // mostly keep the CUs busy (19 single tokens and a piece of 200 to 300: of one
    // batch 46.9, and 52.6 in blocks of 64, of another 45.5 and 41.1).
    auto block_rows = [](int64_t R, bool wide) { return wide && R > 64 ? 128 : 64; };
    auto blocks_with = [&](bool wide) {
        std::vector<Block> v;
        for (int s = 0; s < n_seqs; ++s) {
            const int64_t R = (int64_t)n_new[s] * group;
            if (R <= paged::kFewRows) continue;
            const int rows = block_rows(R, wide);
            for (int64_t r0 = 0; r0 < R; r0 += rows) {
                const int64_t last = std::min(r0 + rows, R);
                v.push_back(Block{(int)((pos0[s] + (last - 1) / group + paged::kStep) / paged::kStep), (int)(last - r0), 1});
            }
        }
        return v;
    };
    const double few_bytes = (double)kFewStep * c.head_dim * (c.flags & ATTN_PAGED_E4M3 ? 2 : 4);   // of a step
    double few_us = 0.0;
    for (int s = 0; s < n_seqs; ++s)
        if (n_new[s] > 0 && (int64_t)n_new[s] * group <= paged::kFewRows)
            few_us += ((int64_t)pos0[s] + n_new[s]) * G * few_bytes / kFewStep / kStreamRate;
    std::vector<Block> blocks = blocks_with(true);
    bool wide = false;
    for (const Block& bl : blocks) wide |= bl.rows > 64;
    const double us = divide_blocks(blocks, G, c.head_dim, wide, few_us);
    if (wide && few_us == 0.0) {
        std::vector<Block> narrow = blocks_with(false);
        if (divide_blocks(narrow, G, c.head_dim, false, few_us) < us) {
            blocks = std::move(narrow);
            wide = false;
        }
    }
    std::vector<int> cuts;
    std::vector<Item> whole;                             // of few()
    size_t block = 0;                                    // the sequence's first of `blocks`
    int few_slot = 0, tile_slot = 0, tok0 = 0, table = 0;
    for (int s = 0; s < n_seqs; ++s) {
        const int R = n_new[s] * group, n_pos = pos0[s] + n_new[s];
        Item it{};
        it.tok0 = tok0;
        it.pos0 = pos0[s];
        it.n_pos = n_pos;
        it.table = table;
        it.holes = holes[s];
        if (R > 0 && R <= paged::kFewRows) {
            it.rows = R;
            it.end = n_pos;
            it.slot = it.next = -1;
            for (it.kvh = 0; it.kvh < G; ++it.kvh) whole.push_back(it);
        } else if (R > 0) {
            const int rows = block_rows(R, wide), kind = rows == 64, n_blocks = (R + rows - 1) / rows;
            for (it.kvh = 0; it.kvh < G; ++it.kvh)
                for (int k = 0; k < n_blocks; ++k) {
                    const Block& bl = blocks[block + k];
                    const int n = bl.ranges;
                    it.row0 = k * rows;
                    it.rows = bl.rows;
                    it.begin = 0;
                    it.end = pos0[s] + (it.row0 + it.rows - 1) / group + 1;
                    if (n > 1) {
                        b.tile_merge.push_back(Merge{tok0, it.row0, it.rows, it.kvh, tile_slot, n, {}});
                        b.slots[1] = std::max(b.slots[1], n);
                    }
                    even_cuts(bl.steps, n, cuts);
                    add_ranges(b.tile[kind], it, cuts, paged::kStep, tile_slot);
                }
            block += n_blocks;
        }
        tok0 += n_new[s];
        table += n_new[s] > 0 ? blocks_of(s) : 0;
    }
    divide_few(whole, few_bytes, b, few_slot);
    b.all_slots[0] = few_slot;
    b.all_slots[1] = tile_slot;
    by_xcd(b.tile[0]);
    by_xcd(b.tile[1]);
}

paged::Args layer_args(attn_paged_ctx* c, int layer)
{
    const Layout& L = c->L;
    paged::Args a{};
    a.hdr = reinterpret_cast<const paged::Header*>(c->ws + L.hdr);
    a.freq = reinterpret_cast<const double*>(c->ws + L.freq);
    a.tok = reinterpret_cast<const paged::Token*>(c->ws + L.tok);
    a.pages = reinterpret_cast<const paged::PageWork*>(c->ws + L.pages);
    a.few = reinterpret_cast<const Item*>(c->ws + L.few);
    for (int k = 0; k < 2; ++k) a.tile[k] = reinterpret_cast<const Item*>(c->ws + L.tile[k]);
    for (int k = 0; k < 2; ++k) a.merge[k] = reinterpret_cast<const Merge*>(c->ws + L.merge[k]);
    a.table = reinterpret_cast<const int32_t*>(c->ws + L.table);
    a.few_part = reinterpret_cast<float*>(c->ws + L.few_part);
    a.tile_part = reinterpret_cast<float*>(c->ws + L.tile_part);
    uint8_t* base = c->cache + (size_t)layer * L.layer_bytes;
    a.k = base;
    a.v = base + L.data_bytes;
    a.k_scale = reinterpret_cast<float*>(base + 2 * L.data_bytes);
    a.v_scale = reinterpret_cast<float*>(base + 2 * L.data_bytes + L.scale_bytes);
    a.T = c->T;
    a.H = c->cfg.n_heads;
    a.G = c->cfg.n_kv_heads;
    a.hd = c->cfg.head_dim;
    a.shift = L.shift;
    a.e4m3 = (c->cfg.flags & ATTN_PAGED_E4M3) != 0;
    return a;
}

// Waits until the stage's last batch has left it, and makes it large enough.
hipError_t ready(Stage& st, size_t bytes)
{
    hipError_t e = hipSuccess;
    if (st.busy) {
        e = hipEventSynchronize(st.done);
        if (e != hipSuccess) return e;
        st.busy = false;
    }
    if (!st.done) {
        e = hipEventCreateWithFlags(&st.done, hipEventDisableTiming);
        if (e != hipSuccess) { st.done = nullptr; return e; }
    }
    if (st.bytes < bytes) {
        if (st.mem) (void)hipHostFree(st.mem);
        st.mem = nullptr;
        st.bytes = 0;
        void* p = nullptr;
        const size_t want = align_up(bytes + bytes / 2, 4096);
        e = hipHostMalloc(&p, want, hipHostMallocDefault);
        if (e != hipSuccess) return e;
        st.mem = static_cast<uint8_t*>(p);
        st.bytes = want;
    }
    return hipSuccess;
}

moe_status check_call(attn_paged_ctx* ctx, int32_t layer)
{
    if (layer < 0 || layer >= ctx->cfg.n_layers) return fail(ctx, MOE_E_ARG, "layer out of range");
    if (!ctx->set) return fail(ctx, MOE_E_STATE, "no batch set");
    return MOE_OK;
}

bool capturing(hipStream_t s)
{
    hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
    return hipStreamIsCapturing(s, &st) == hipSuccess && st != hipStreamCaptureStatusNone;
}

moe_status set_batch(attn_paged_ctx* ctx, int32_t n_seqs, const int32_t* n_new, const int32_t* pos0,
                     const int32_t* table, int32_t ld, hipStream_t s)
{
    const attn_paged_config& c = ctx->cfg;
    const Layout& L = ctx->L;
    if (n_seqs < 0) return fail(ctx, MOE_E_ARG, "n_seqs is negative");
    if (n_seqs > c.max_seqs) return fail(ctx, MOE_E_CAPACITY, "n_seqs exceeds max_seqs");
    if (n_seqs > 0 && (!n_new || !pos0 || !table)) return fail(ctx, MOE_E_ARG, "n_new, pos0 or table is NULL");
    if (n_seqs > 0 && ld < 1) return fail(ctx, MOE_E_ARG, "ld must be at least 1");
    int64_t T = 0;
    for (int i = 0; i < n_seqs; ++i) {
        if (n_new[i] < 0 || pos0[i] < 0) return fail(ctx, MOE_E_ARG, "n_new and pos0 must be non-negative");
        T += n_new[i];
    }
    if (T > c.max_tokens) return fail(ctx, MOE_E_CAPACITY, "the batch's tokens exceed max_tokens");
    Batch b;
    std::vector<uint8_t> holes(n_seqs, 0);
    b.tok.reserve(T);
    if (ctx->call == INT32_MAX) {
        std::fill(ctx->written.begin(), ctx->written.end(), 0);
        ctx->call = 0;
    }
    const int32_t call = ++ctx->call;
    for (int i = 0; i < n_seqs; ++i) {
        const int64_t n_pos = (int64_t)pos0[i] + n_new[i], blocks = (n_pos + c.page_size - 1) >> L.shift;
        if (blocks > c.max_blocks) return fail(ctx, MOE_E_CAPACITY, "a sequence exceeds max_blocks pages");
        if (blocks > ld) return fail(ctx, MOE_E_ARG, "ld is smaller than a sequence's pages");
        const int32_t* row = table + (int64_t)i * ld;
        for (int64_t k = 0; k < blocks; ++k) {
            if (row[k] < -1 || row[k] >= c.n_pages) return fail(ctx, MOE_E_ARG, "a table entry is outside -1 .. n_pages - 1");
            if (row[k] < 0) holes[i] = 1;
        }
        if (n_new[i] == 0) continue;
        b.table.insert(b.table.end(), row, row + blocks);
        for (int64_t k = pos0[i] >> L.shift; k < blocks; ++k) {
            const int32_t page = row[k];
            if (page >= 0 && ctx->written[page] == call) return fail(ctx, MOE_E_ARG, "a page would be written twice");
            if (page >= 0) ctx->written[page] = call;
            else b.unplaced = true;
            const int64_t lo = std::max<int64_t>(pos0[i], k << L.shift), hi = std::min(n_pos, (k + 1) << L.shift);
            if (page >= 0)
                b.pages.push_back(paged::PageWork{page, (int32_t)(lo - (k << L.shift)), (int32_t)(hi - lo), (int32_t)b.tok.size()});
            for (int64_t p = lo; p < hi; ++p) b.tok.push_back(paged::Token{(int32_t)p, page});
        }
    }
    divide(c, L, n_new, pos0, n_seqs, holes, b);
    if (b.few.size() > L.max_few || b.tile[0].size() > L.max_tile[0] || b.tile[1].size() > L.max_tile[1] ||
        b.merge.size() > L.max_merge[0] || b.tile_merge.size() > L.max_merge[1] ||
        (size_t)b.all_slots[0] > L.few_slots || (size_t)b.all_slots[1] > L.tile_slots)
        return fail(ctx, MOE_E_CAPACITY, "the batch has more shares than the workspace holds");
    // (no tokens: nothing is launched, but a graph of an earlier batch that is
    // replayed all the same must find so)
    if (T > 0 || ctx->handed) {
        paged::Header h{};
        h.T = (int32_t)T;
        h.n_pages = (int32_t)b.pages.size();
        h.n_few = b.n_runs;
        for (int k = 0; k < 2; ++k) h.n_tile[k] = (int32_t)b.tile[k].size();
        h.n_merge[0] = (int32_t)b.merge.size();
        h.n_merge[1] = (int32_t)b.tile_merge.size();
        const struct { size_t dst; const void* src; size_t bytes; } parts[paged::kSegments] = {
            {L.hdr, &h, sizeof h},
            {L.freq, ctx->freq.data(), ctx->freq.size() * 8},
            {L.tok, b.tok.data(), b.tok.size() * sizeof(paged::Token)},
            {L.pages, b.pages.data(), b.pages.size() * sizeof(paged::PageWork)},
            {L.few, b.few.data(), b.few.size() * sizeof(Item)},
            {L.tile[0], b.tile[0].data(), b.tile[0].size() * sizeof(Item)},
            {L.tile[1], b.tile[1].data(), b.tile[1].size() * sizeof(Item)},
            {L.merge[0], b.merge.data(), b.merge.size() * sizeof(Merge)},
            {L.merge[1], b.tile_merge.data(), b.tile_merge.size() * sizeof(Merge)},
            {L.table, b.table.data(), b.table.size() * 4}};
        size_t bytes = 0;
        for (const auto& p : parts) bytes += align_up(p.bytes, 16);
        if (capturing(s)) return fail(ctx, MOE_E_STATE, "a batch cannot be set while the stream captures a graph");
        ctx->set = false;                                // (until the new one is on its way)
        Stage& st = ctx->stage[ctx->next_stage];
        hipError_t e = ready(st, bytes);
        if (e != hipSuccess) return hip_fail(ctx, e, "pinned memory for the batch");
        paged::Unpack u{};
        u.src = st.mem;
        u.dst = ctx->ws;
        size_t at = 0;
        for (int k = 0; k < paged::kSegments; ++k) {
            const size_t n = align_up(parts[k].bytes, 16);
            if (parts[k].bytes) std::memcpy(st.mem + at, parts[k].src, parts[k].bytes);
            if (n > parts[k].bytes) std::memset(st.mem + at + parts[k].bytes, 0, n - parts[k].bytes);
            u.seg[k] = paged::Segment{parts[k].dst, at};
            at += n;
        }
        u.bytes = at;
        ctx->handed = true;
        e = attn_paged_launch_unpack(&u, s);
        if (e != hipSuccess) return hip_fail(ctx, e, "batch kernel launch");
        e = hipEventRecord(st.done, s);
        if (e != hipSuccess) {
            (void)hipStreamSynchronize(s);               // nothing else tells when the stage has been read
            return hip_fail(ctx, e, "batch event");
        }
        st.busy = true;
        ctx->next_stage = (ctx->next_stage + 1) % kStages;
        ctx->handed = T > 0;
    }
    ctx->T = (int32_t)T;
    ctx->n_pages = (int32_t)b.pages.size();
    ctx->n_few = b.n_runs;
    for (int k = 0; k < 2; ++k) ctx->n_tile[k] = (int32_t)b.tile[k].size();
    ctx->n_merge[1] = (int32_t)b.tile_merge.size();
    ctx->n_merge[0] = (int32_t)b.merge.size();
    for (int k = 0; k < 2; ++k) ctx->slots[k] = b.slots[k];
    ctx->unplaced = b.unplaced;
    ctx->set = true;
    return MOE_OK;
}

}  // namespace

extern "C" {

int32_t attn_paged_tokens(const attn_paged_ctx* ctx) { return ctx->T; }
const attn_paged_config* attn_paged_cfg(const attn_paged_ctx* ctx) { return &ctx->cfg; }
int attn_paged_can_append(const attn_paged_ctx* ctx) { return ctx->set && !ctx->unplaced; }

hipError_t attn_paged_run_append(attn_paged_ctx* ctx, int32_t layer, const paged::Source* x, uint16_t* q,
                                 hipStream_t s)
{
    const paged::Args a = layer_args(ctx, layer);
    return attn_paged_launch_append(&a, x, q, ctx->T, ctx->n_pages, s);
}

hipError_t attn_paged_run_attend(attn_paged_ctx* ctx, int32_t layer, const uint16_t* q, uint16_t* out,
                                 hipStream_t s)
{
    const paged::Args a = layer_args(ctx, layer);
    // A graph may replay on a longer batch: its launches have room for the
    // shares that one may have, of row blocks of either kind, and the merge is
    // there (its entries: a sequence's and key/value head's rows, a row block's).
    const bool graph = capturing(s);
    int n[3] = {ctx->n_few, ctx->n_tile[0], ctx->n_tile[1]};
    int m[2] = {ctx->n_merge[0], ctx->n_merge[1]}, slots[2] = {ctx->slots[0], ctx->slots[1]};
    if (graph) {
        if (n[0]) n[0] = std::max(n[0], kGraphGrid);
        if (n[1] || n[2])
            for (int k = 1; k <= 2; ++k) n[k] = std::max(n[k], kGraphGrid);
        m[0] = n[0] ? std::max(m[0], kGraphMerge) : 0;
        m[1] = n[1] || n[2] ? std::max(m[1], kGraphMerge) : 0;
        slots[0] = slots[1] = INT32_MAX;
    }
    const hipError_t e = attn_paged_launch_attend(&a, q, out, n, s);
    if (e != hipSuccess || (m[0] == 0 && m[1] == 0)) return e;
    return attn_paged_launch_merge(&a, out, m, slots, paged::kFewRows, s);
}

size_t attn_paged_cache_bytes(const attn_paged_config* cfg)
{
    return check_config(cfg) ? 0 : make_layout(cfg).cache_bytes;
}

size_t attn_paged_workspace_bytes(const attn_paged_config* cfg)
{
    return check_config(cfg) ? 0 : make_layout(cfg).ws_bytes;
}

moe_status attn_paged_init(const attn_paged_config* cfg, void* cache, void* workspace, attn_paged_ctx** out)
{
    if (!out) return fail(nullptr, MOE_E_ARG, "out is NULL");
    *out = nullptr;
    if (const char* why = check_config(cfg)) return fail(nullptr, MOE_E_SHAPE, why);
    if (!cache || !workspace) return fail(nullptr, MOE_E_ARG, "cache or workspace is NULL");
    if (((uintptr_t)cache | (uintptr_t)workspace) & (kAlign - 1))
        return fail(nullptr, MOE_E_ALIGN, "cache and workspace must be 256-byte aligned");
    attn_paged_ctx* c = new (std::nothrow) attn_paged_ctx();
    if (!c) return fail(nullptr, MOE_E_ARG, "out of host memory");
    c->cfg = *cfg;
    c->L = make_layout(cfg);
    c->cache = static_cast<uint8_t*>(cache);
    c->ws = static_cast<uint8_t*>(workspace);
    try {
        c->freq.resize(cfg->head_dim / 2);
        c->written.assign(cfg->n_pages, 0);
    } catch (...) {
        delete c;
        return fail(nullptr, MOE_E_ARG, "out of host memory");
    }
    for (int f = 0; f < cfg->head_dim / 2; ++f) c->freq[f] = std::pow((double)cfg->rope_theta, -2.0 * f / cfg->head_dim);
    *out = c;
    return MOE_OK;
}

moe_status attn_paged_set_batch(attn_paged_ctx* ctx, int32_t n_seqs, const int32_t* n_new, const int32_t* pos0,
                                const int32_t* table, int32_t ld, moe_stream_t stream)
{
    if (!ctx) return MOE_E_ARG;
    try {
        return set_batch(ctx, n_seqs, n_new, pos0, table, ld, static_cast<hipStream_t>(stream));
    } catch (...) {
        return fail(ctx, MOE_E_ARG, "out of host memory for the batch");
    }
}

moe_status attn_paged_append(attn_paged_ctx* ctx, int32_t layer, const void* qkv, int64_t ld, int32_t type,
                             uint16_t* q, moe_stream_t stream)
{
    if (!ctx) return MOE_E_ARG;
    const moe_status st = check_call(ctx, layer);
    if (st != MOE_OK) return st;
    const attn_paged_config& c = ctx->cfg;
    if (type != ATTN_QKV_F32 && type != ATTN_QKV_BF16) return fail(ctx, MOE_E_ARG, "unknown type of q | k | v");
    const int64_t n = (int64_t)(c.n_heads + 2 * c.n_kv_heads) * c.head_dim;
    if (ld < n || ld > (INT64_MAX >> 20)) return fail(ctx, MOE_E_ARG, "ld is smaller than a row of q | k | v, or too large");
    if (ld % (type == ATTN_QKV_BF16 ? 8 : 4)) return fail(ctx, MOE_E_ALIGN, "the rows of q | k | v must be 16-byte aligned");
    if (ctx->unplaced) return fail(ctx, MOE_E_STATE, "a new token of the batch has no page");
    if (ctx->T == 0) return MOE_OK;
    if (!qkv || !q) return fail(ctx, MOE_E_ARG, "qkv or q is NULL");
    if (misaligned(qkv) || misaligned(q)) return fail(ctx, MOE_E_ALIGN, "qkv and q must be 16-byte aligned");
    const uint64_t qkv_bytes = ((uint64_t)(ctx->T - 1) * ld + n) * (type == ATTN_QKV_BF16 ? 2 : 4);
    if (overlap(qkv, qkv_bytes, q, q_bytes(ctx))) return fail(ctx, MOE_E_ARG, "q may not overlap qkv");
    const paged::Source x{qkv, ld, 0, 1, type == ATTN_QKV_BF16, 0};
    const hipError_t e = attn_paged_run_append(ctx, layer, &x, q, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(ctx, e, "append kernel launch");
    return MOE_OK;
}

moe_status attn_paged_attend(attn_paged_ctx* ctx, int32_t layer, const uint16_t* q, uint16_t* out,
                             moe_stream_t stream)
{
    if (!ctx) return MOE_E_ARG;
    const moe_status st = check_call(ctx, layer);
    if (st != MOE_OK) return st;
    if (ctx->T == 0) return MOE_OK;
    if (!q || !out) return fail(ctx, MOE_E_ARG, "q or out is NULL");
    if (overlap(q, q_bytes(ctx), out, q_bytes(ctx))) return fail(ctx, MOE_E_ARG, "out may not overlap q");
    if (misaligned(q) || misaligned(out)) return fail(ctx, MOE_E_ALIGN, "q and out must be 16-byte aligned");
    const hipError_t e = attn_paged_run_attend(ctx, layer, q, out, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(ctx, e, "attention kernel launch");
    return MOE_OK;
}

void attn_paged_destroy(attn_paged_ctx* ctx)
{
    if (!ctx) return;
    for (Stage& st : ctx->stage) {
        if (st.busy) (void)hipEventSynchronize(st.done);
        if (st.done) (void)hipEventDestroy(st.done);
        if (st.mem) (void)hipHostFree(st.mem);
    }
    delete ctx;
}

const char* attn_paged_last_error(const attn_paged_ctx* ctx) { return ctx ? ctx->err.c_str() : g_init_error.c_str(); }

}  // extern "C"
