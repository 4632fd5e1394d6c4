// Divides random batches as attn_paged_set_batch does and checks the shares: every position of
// every row exactly once, runs that end, partial sums of their own that the merge lists name, all
// within the workspace.  Built on the host alone, the kernels' launchers being stubs.
// usage: paged_divide SEED BATCHES
#include "../paper_2506_23635_amd/csrc/attn_paged_capi.cpp"

#include <array>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>

extern "C" {
hipError_t attn_paged_launch_unpack(const paged::Unpack*, hipStream_t) { return hipErrorUnknown; }
hipError_t attn_paged_launch_append(const paged::Args*, const paged::Source*, uint16_t*, int, int, hipStream_t) { return hipErrorUnknown; }
hipError_t attn_paged_launch_attend(const paged::Args*, const uint16_t*, uint16_t*, const int*, hipStream_t) { return hipErrorUnknown; }
hipError_t attn_paged_launch_merge(const paged::Args*, uint16_t*, const int*, const int*, int, hipStream_t) { return hipErrorUnknown; }
}

static int n_batch;
#define CHECK(...)                                                                                   \
    do {                                                                                             \
        if (!(__VA_ARGS__)) {                                                                        \
            std::printf("batch %d, line %d: %s\n", n_batch, __LINE__, #__VA_ARGS__);                 \
            std::exit(1);                                                                            \
        }                                                                                            \
    } while (0)

typedef std::array<int, 3> Key;            // first token, key/value head, first row

// The shares of one block of rows cover positions 0 .. end - 1 in order, with the merge's slots.
static void check_rows(std::vector<Item> v, int end, int step, const std::map<Key, Merge>& merges, Key key)
{
    std::sort(v.begin(), v.end(), [](const Item& x, const Item& y) { return x.begin < y.begin; });
    const bool several = v.size() > 1;
    CHECK(merges.count(key) == (several ? 1u : 0u));
    int at = 0;
    for (size_t k = 0; k < v.size(); ++k) {
        CHECK(v[k].begin == at && v[k].end > at && at % step == 0 && v[k].rows == v[0].rows);
        at = v[k].end;
        if (!several) {
            CHECK(v[k].slot == -1);
            continue;
        }
        const Merge& m = merges.at(key);
        CHECK(m.n == (int)v.size() && m.rows == v[0].rows && v[k].slot == m.slot0 + (int)k);
    }
    CHECK(at == end);
}

static std::map<Key, Merge> slots_of(const std::vector<Merge>& list, int most, int all_slots)
{
    std::map<Key, Merge> by;
    std::set<int> used;
    for (const Merge& m : list) {
        CHECK(m.n >= 2 && m.n <= most);
        CHECK(by.emplace(Key{m.tok0, m.kvh, m.row0}, m).second);
        for (int k = 0; k < m.n; ++k) CHECK(m.slot0 + k >= 0 && m.slot0 + k < all_slots && used.insert(m.slot0 + k).second);
    }
    return by;
}

int main(int argc, char** argv)
{
    std::mt19937 rng(argc > 1 ? std::atoi(argv[1]) : 1);
    const int batches = argc > 2 ? std::atoi(argv[2]) : 1000;
    auto R = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    int divided[2] = {0, 0};
    for (n_batch = 0; n_batch < batches; ++n_batch) {
        static const int heads[] = {1, 2, 4, 8, 16, 64}, groups[] = {1, 2, 6, 8, 16};
        attn_paged_config c{};
        c.n_kv_heads = heads[R(0, 5)];
        c.n_heads = c.n_kv_heads * groups[R(0, 4)];
        c.head_dim = R(0, 1) ? 64 : 128;
        c.page_size = 16 << R(0, 4);
        c.n_pages = c.n_layers = 1;
        c.max_blocks = std::min(R(0, 2) ? R(1, 500) : R(1, 65536), (1 << 24) / c.page_size);
        const int S = c.max_seqs = R(0, 3) == 0 ? R(1, 3) : R(0, 9) ? R(1, 70) : R(1, 700);
        c.rope_theta = 5e5f;
        c.flags = R(0, 1);
        std::vector<int32_t> n(S), p(S);
        const int mode = R(0, 3), room = c.max_blocks * c.page_size;
        int T = 0;
        for (int s = 0; s < S; ++s) {
            n[s] = std::min(room, mode < 2 ? 1 : mode == 2 ? R(0, 4) : R(0, 9) ? R(0, 2) : R(0, 2000));
            if (T + n[s] > 32768) n[s] = 0;
            T += n[s];
            p[s] = std::min(room - n[s], R(0, 3) ? R(0, room) : R(0, 300));
        }
        if (T == 0) continue;
        c.max_tokens = std::min(32768, T + R(0, 5));
        if (check_config(&c)) continue;
        const Layout L = make_layout(&c);
        Batch b;
        divide(c, L, n.data(), p.data(), S, std::vector<uint8_t>(S, 0), b);

        CHECK(b.few.size() <= L.max_few && b.merge.size() <= L.max_merge[0] && (size_t)b.all_slots[0] <= L.few_slots);
        CHECK(b.tile_merge.size() <= L.max_merge[1] && (size_t)b.all_slots[1] <= L.tile_slots);
        // (a launch's workgroups, a multiple of eight, each read the list's entry of their number)
        CHECK(b.few.empty() || (size_t)std::max(b.n_runs, kGraphGrid) + kXcds <= L.max_few);
        for (int k = 0; k < 2; ++k)
            CHECK(std::max(b.tile[k].size(), (size_t)(b.tile[0].size() + b.tile[1].size() ? kGraphGrid : 0)) + kXcds <= L.max_tile[k] ||
                  b.tile[0].size() + b.tile[1].size() == 0);
        divided[0] += !b.merge.empty();
        divided[1] += !b.tile_merge.empty();

        std::map<Key, std::vector<Item>> rows;
        std::vector<char> seen(b.few.size(), 0);
        CHECK(b.n_runs <= (int)b.few.size());
        for (int r = 0; r < b.n_runs; ++r)
            for (int i = r; i >= 0; i = b.few[i].next) {
                CHECK(i < (int)b.few.size() && !seen[i] && (i == r || i >= b.n_runs));
                seen[i] = 1;
                rows[Key{b.few[i].tok0, b.few[i].kvh, -1}].push_back(b.few[i]);
            }
        for (char s : seen) CHECK(s);
        for (int k = 0; k < 2; ++k)
            for (const Item& x : b.tile[k]) {
                CHECK(x.rows >= 1 && x.rows <= 128 >> k && x.row0 % (128 >> k) == 0);
                rows[Key{x.tok0, x.kvh, x.row0}].push_back(x);
            }
        std::map<Key, Merge> few_merges = slots_of(b.merge, paged::kFewRuns, b.all_slots[0]);
        const std::map<Key, Merge> tile_merges = slots_of(b.tile_merge, 16, b.all_slots[1]);
        size_t blocks = 0, tok0 = 0;
        for (int s = 0; s < S; tok0 += n[s++]) {
            const int group = c.n_heads / c.n_kv_heads, count = n[s] * group;
            for (int g = 0; g < c.n_kv_heads && count > 0; ++g) {
                if (count <= paged::kFewRows) {
                    const Key key{(int)tok0, g, -1};
                    CHECK(rows.count(key) && rows[key][0].rows == count && rows[key][0].pos0 == p[s] && rows[key][0].n_pos == p[s] + n[s]);
                    std::map<Key, Merge> m;
                    if (few_merges.count(Key{(int)tok0, g, 0})) m[key] = few_merges[Key{(int)tok0, g, 0}];
                    check_rows(rows[key], p[s] + n[s], kFewStep, m, key);
                    ++blocks;
                    continue;
                }
                for (int r0 = 0; r0 < count; ++blocks) {
                    const Key key{(int)tok0, g, r0};
                    CHECK(rows.count(key) && rows[key][0].pos0 == p[s] && rows[key][0].n_pos == p[s] + n[s]);
                    const int end = r0 + rows[key][0].rows;
                    check_rows(rows[key], p[s] + (end - 1) / group + 1, paged::kStep, tile_merges, key);
                    r0 = end;
                }
            }
        }
        CHECK(blocks == rows.size());
    }
    std::printf("%d %d\n", divided[0], divided[1]);
    return 0;
}
