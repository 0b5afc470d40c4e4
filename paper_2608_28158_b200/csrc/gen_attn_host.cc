// Host index for the attention of sampled tokens on the cached tree: which queries see which tokens of a node, cut into units of
// work (rows x a run of tokens) for the two kernels, and where the parts of a query's sum are.
//
// A node's tokens are seen by its own queries, up to their positions, and by those of every branch below a fork, up to the fork.  Runs of tokens
// between such limits are read once for all queries that see them; limits that lie within MIXED tokens of each other are taken
// together, and the narrow kernel then looks at every row's own limit.  A node that only its own queries see is one run.
#include <algorithm>
#include <cstdint>
#include <new>
#include <utility>
#include <vector>

#include "gen.h"

namespace {

using namespace harts::gen_attn;

constexpr int TILE = 64;
constexpr int MIXED = 2 * TILE;         // limits this near to each other share a run
constexpr int LEAST = 256;              // tokens a wide unit is not cut below
constexpr int START = 20 * TILE;        // tokens that it counts for besides its own: queries, outputs and the merge of its parts
constexpr int SMS = 148;
constexpr int PIECE = 2;                // tiles that are not cut off a narrow unit
// Tiles that a narrow unit costs besides its own: its rows, queries and first page follow each other.  Counted as two, a list of short units took twice
// as long as the others: 64 sequences of 2,600 tokens with a branch of 16 and two drafts each, 8 bits, 103 us, 60 with five; 30 of 8,000 68 and 52.
constexpr int UNIT = 5;
// Below so many tokens (one short unit an SM, all key heads) a call's time is the kernels' latency, and the narrow kernel's is the shorter:
// 28 rows x 700 tokens 12.4 against 16.4 us.  Above, from 16 rows on the wide one (agentic trees, 32 rows x 900: 92 against 119 us).
constexpr int64_t SMALL = SMS * 256;
constexpr int SMALL_ROWS = 32;

constexpr size_t MAX_ENTRIES = (size_t)INT32_MAX / (sizeof(Entry) / 4);        // more do not fit into the index

struct Range {
    int node, a, b, entry, n_entries;
    bool wide;
};
struct Index {
    std::vector<Unit> narrow, wide;
    std::vector<Entry> entries;
    std::vector<int32_t> part_ptr, part, list_ptr;
    int32_t n_parts = 0, merged = 0, max_page = -1;
};

bool forest_ok(int32_t n_trees, const int32_t* ptr, const int32_t* parent, const int32_t* off, const int32_t* len) {
    for (int32_t t = 0; t < n_trees; t++) {
        const int32_t lo = ptr[t], hi = ptr[t + 1];
        for (int32_t i = lo; i < hi; i++) {
            if (len[i] < 0) return false;
            if (i == lo ? (parent[i] != -1 || off[i] != 0) : (parent[i] < 0 || parent[i] >= i - lo || off[i] < 0 || off[i] > len[lo + parent[i]])) return false;
        }
    }
    return true;
}

int32_t build(int32_t n_trees, const int32_t* ptr, const int32_t* parent, const int32_t* off, const int32_t* len, const int32_t* page_ptr,
              const int32_t* pages, int32_t page, int32_t n_q, const int32_t* q_node, const int32_t* q_pos, int32_t Hq, int32_t Hkv, int32_t grow,
              Index& ix) {
    const int32_t n_nodes = ptr[n_trees], G = Hq / Hkv;
    struct Sees {
        int32_t row, limit;              // -1: its own node
    };
    std::vector<std::vector<Sees>> sees(n_nodes);
    std::vector<int32_t> base(n_nodes);
    for (int32_t t = 0; t < n_trees; t++)
        for (int32_t i = ptr[t]; i < ptr[t + 1]; i++) base[i] = ptr[t];
    for (int32_t r = 0; r < n_q; r++) {
        if (q_node[r] < 0) continue;
        if (q_node[r] >= n_nodes || q_pos[r] < -1 || q_pos[r] >= len[q_node[r]]) return HARTS_EINVAL;
        int32_t v = q_node[r];
        sees[v].push_back({r, -1});
        for (; parent[v] >= 0; v = base[v] + parent[v])
            if (off[v] > 0) sees[base[v] + parent[v]].push_back({r, off[v]});
    }
    int64_t tokens = 0;
    for (int32_t v = 0; v < n_nodes; v++) tokens += sees[v].empty() ? 0 : len[v];
    const int64_t most_rows = tokens * Hkv < SMALL ? SMALL_ROWS : NARROW_ROWS;
    std::vector<Range> ranges;
    auto add = [&](int node, int a, int b, bool wide, const std::vector<Entry>& e) {
        if (e.empty() || b <= a || ix.entries.size() >= MAX_ENTRIES) return;
        ranges.push_back({node, a, b, (int)ix.entries.size(), (int)e.size(), wide && (int64_t)e.size() * G > most_rows});
        ix.entries.insert(ix.entries.end(), e.begin(), e.end());
    };
    std::vector<Entry> e;
    for (int32_t v = 0; v < n_nodes; v++) {
        auto& s = sees[v];
        int n_own = 0;
        int64_t least = INT32_MAX;
        for (const Sees& x : s)
            if (x.limit < 0) {
                n_own++;
                least = std::min<int64_t>(least, q_pos[x.row] + 1);
            }
        const int64_t room = ((int64_t)page_ptr[v + 1] - page_ptr[v]) * page, most = std::min<int64_t>((int64_t)len[v] + (n_own ? grow : 0), room);
        if (room < len[v] || most >= INT32_MAX - (1 << 16)) return HARTS_EINVAL;
        for (int32_t p = page_ptr[v]; p < page_ptr[v + 1]; p++) {
            if (pages[p] < 0) return HARTS_EINVAL;
            ix.max_page = std::max(ix.max_page, pages[p]);
        }
        if (s.empty()) continue;
        // what its own queries see for certain, in whole tiles and without the last token, is shared with the branches below; a node of few rows alone is one run
        int own_from = 0;
        if (n_own && (n_own < (int)s.size() || (int64_t)n_own * G > NARROW_ROWS)) own_from = least > 0 ? (int)((least - 1) / TILE * TILE) : 0;
        std::vector<int32_t> limits;
        for (Sees& x : s) {
            const int32_t l = x.limit < 0 ? own_from : x.limit;
            if (l > 0) limits.push_back(l);
        }
        std::sort(limits.begin(), limits.end());
        limits.erase(std::unique(limits.begin(), limits.end()), limits.end());
        auto seeing = [&](int from, int to) {           // queries that see tokens behind `from`, up to `to` at most
            e.clear();
            for (const Sees& x : s) {
                const int32_t l = x.limit < 0 ? own_from : x.limit;
                if (l > from) e.push_back({x.row, std::min(l, to), 0, 0});
            }
        };
        int a = 0;
        for (size_t i = 0; i < limits.size();) {
            if (limits[i] - a > MIXED || i + 1 == limits.size()) {
                seeing(a, limits[i]);
                add(v, a, limits[i], true, e);
                a = limits[i++];
                continue;
            }
            size_t j = i;
            while (j + 1 < limits.size() && limits[j + 1] - a <= MIXED) j++;
            seeing(a, limits[j]);
            add(v, a, limits[j], j == i, e);
            a = limits[j];
            i = j + 1;
        }
        if (n_own) {
            e.clear();
            for (const Sees& x : s)
                if (x.limit < 0) e.push_back({x.row, -1, q_pos[x.row] + 1, (int32_t)most});
            add(v, own_from, (int)most, false, e);
        }
    }
    if (ix.entries.size() >= MAX_ENTRIES) return HARTS_EINVAL;
    // Rows of a narrow unit: eight where no run of few rows has more (the kernel is the faster of the two).
    auto tiles_of = [](int a, int b) { return (int64_t)(b + TILE - 1) / TILE - a / TILE; };
    int block_rows = 8;
    for (const Range& r : ranges)
        if (!r.wide && (int64_t)r.n_entries * G > 8) block_rows = NARROW_ROWS;
    if (G > 8) block_rows = NARROW_ROWS;
    // A little wide work beside much narrow work costs more as a kernel of its own than as blocks of few rows that read its tokens again
    // (64 branches of 1,300 tokens on a prompt of 64: 52 -> 43 us).
    auto blocks = [&](const Range& r, int rows) { return ((int64_t)r.n_entries * G + rows - 1) / rows; };
    int64_t narrow_tiles = 0, wide_tiles = 0, again = 0;
    for (const Range& r : ranges)
        if (r.wide) {
            wide_tiles += blocks(r, WIDE_ROWS) * tiles_of(r.a, r.b);
            again += blocks(r, block_rows) * tiles_of(r.a, r.b);
        } else {
            narrow_tiles += blocks(r, block_rows) * tiles_of(r.a, r.b);
        }
    if (8 * again <= narrow_tiles) {
        for (Range& r : ranges) r.wide = false;
        wide_tiles = 0;
    }
    // Much of both: one CTA of either kernel on an SM, products of the one under the memory traffic of the other (64 branches on a prompt of
    // 16,421 tokens, 28 wide and 38 narrow tiles an SM: 80 -> 61 us).  A tile takes such a CTA 1.5 times what it takes the kernel alone, so
    // beyond 2 : 1 they run one after the other, each with the GPU to itself.
    const bool beside = wide_tiles > 0 && narrow_tiles <= 2 * wide_tiles && wide_tiles <= 2 * narrow_tiles;
    std::stable_sort(ranges.begin(), ranges.end(), [](const Range& x, const Range& y) { return x.b - x.a > y.b - y.a; });
    std::vector<std::vector<int32_t>> parts(n_q);
    int64_t n_parts = 0;
    // queries first_entry .. + n of a range, for tokens k0 .. k1, in blocks of `per` rows
    auto put = [&](std::vector<Unit>& to, const Range& r, int first_entry, int n, int per, int k0, int k1) {
        const int rows = n * G;
        for (int f = 0; f < rows; f += per)
            to.push_back({r.entry + first_entry, f, std::min(per, rows - f), k0, k1, page_ptr[r.node], (int32_t)n_parts, 0});
        for (int i = 0; i < n; i++) parts[ix.entries[r.entry + first_entry + i].row].push_back((int32_t)(n_parts + (int64_t)i * G));
        n_parts += rows;
        return n_parts <= INT32_MAX - (1 << 20);
    };

    // The wide kernel's runs are cut into pieces of at most `lo` tokens, by what a length should take: the longest piece where all of them run at
    // once, else a CTA's share and a quarter of the longest piece (the long ones go first).  Against the shortest pieces that run at once,
    // where there are any, and two thirds of a share: agentic trees in bf16, 282 runs of up to 9,000 tokens, 160 -> 71 us; 13 more forests 0 to
    // 20 % less, three 2 to 4 % more.
    int64_t total = 0, most = LEAST;
    for (const Range& r : ranges)
        if (r.wide) {
            total += blocks(r, WIDE_ROWS) * (r.b - r.a) * Hkv;
            most = std::max<int64_t>(most, r.b - r.a);
        }
    const int64_t want = SMS * (beside ? 1 : 2), share = total / want;
    auto estimate = [&](int64_t p) {
        int64_t n = 0, longest = 0;
        for (const Range& r : ranges)
            if (r.wide) {
                const int64_t pieces = (r.b - r.a + p - 1) / p;
                n += blocks(r, WIDE_ROWS) * Hkv * pieces;
                longest = std::max<int64_t>(longest, (r.b - r.a + pieces - 1) / pieces);
            }
        return std::make_pair(n <= want ? longest + START : (total + START * n) / want + longest / 4, n);
    };
    int64_t lo = most, best = total > 0 ? estimate(most).first : 0;
    auto weigh = [&](int64_t p) {
        p = std::min(std::max<int64_t>(p, LEAST), most);
        const int64_t y = estimate(p).first;
        if (y < best) {
            best = y;
            lo = p;
        }
    };
    if (total > 0) {
        for (int i = 2; i <= 12; i++) weigh(share * i / 6);
        int64_t l = LEAST, h = most;              // the shortest pieces that run at once
        while (l < h) {
            const int64_t mid = (l + h) / 2;
            if (estimate(mid).second <= want) h = mid;
            else l = mid + 1;
        }
        weigh(l);
    }
    for (const Range& r : ranges) {
        if (!r.wide) continue;
        const int64_t n = r.b - r.a, pieces = (n + lo - 1) / lo;
        for (int64_t p = 0; p < pieces; p++) {
            auto edge = [&](int64_t i) { return (int32_t)(i <= 0 ? r.a : i >= pieces ? r.b : std::max<int64_t>(r.a, (r.a + n * i / pieces) / TILE * TILE)); };
            if (edge(p + 1) > edge(p) && !put(ix.wide, r, 0, r.n_entries, WIDE_ROWS, edge(p), edge(p + 1))) return HARTS_EINVAL;
        }
    }
    std::stable_sort(ix.wide.begin(), ix.wide.end(), [](const Unit& x, const Unit& y) { return x.k1 - x.k0 > y.k1 - y.k0; });

    // The narrow kernel's: queries in blocks of 8 or 16 rows (a query of more heads is several blocks that are cut alike), and a list for every CTA
    // until its share of the tiles is full; a run that crosses a list's end is cut there.
    const int per_block = std::max(1, block_rows / G);
    int64_t tiles = 0, strips = 0;
    const int chunks = (G + NARROW_ROWS - 1) / NARROW_ROWS;
    for (const Range& r : ranges)
        if (!r.wide) {
            const int64_t n = (r.n_entries + per_block - 1) / per_block * (int64_t)chunks;
            strips += n;
            tiles += n * tiles_of(r.a, r.b);
        }
    if (strips) {
        const int64_t ctas = SMS * (beside ? 1 : block_rows == 8 ? 3 : 2), lists = std::max<int64_t>(1, ctas / Hkv);
        // the lists for a share of tiles: piece(range, first query, queries, from, to) and closed() in order; how many there are
        auto fill = [&](int64_t share, auto piece, auto closed) {
            int64_t full = 0, n_lists = 0;        // full: tiles of the list that is being filled
            auto close = [&]() {
                if (full > 0) {
                    closed();
                    n_lists++;
                }
                full = 0;
            };
            for (const Range& r : ranges) {
                if (r.wide) continue;
                for (int e0 = 0; e0 < r.n_entries; e0 += per_block) {
                    const int n = std::min(per_block, r.n_entries - e0);
                    for (int a = r.a; a < r.b;) {
                        int64_t take = (share - full - UNIT) / chunks;
                        const int64_t left = tiles_of(a, r.b);
                        if (full > 0 && take < std::min<int64_t>(left, PIECE)) {
                            close();
                            take = (share - UNIT) / chunks;
                        }
                        take = std::max<int64_t>(take, 1);
                        const int b = left <= take ? r.b : (int)((a / TILE + take) * TILE);
                        piece(r, e0, n, a, b);
                        full += chunks * (tiles_of(a, b) + UNIT);
                        a = b;
                    }
                }
            }
            close();
            return n_lists;
        };
        // the smallest share that needs no more lists than there are CTAs
        auto none = [](auto&&...) {};
        int64_t lo = std::max<int64_t>((tiles + strips * UNIT) / lists, UNIT + PIECE), hi = lo;
        while (fill(hi, none, none) > lists) hi += hi / 4 + 1;
        while (lo < hi) {
            const int64_t mid = (lo + hi) / 2;
            if (fill(mid, none, none) <= lists) hi = mid;
            else lo = mid + 1;
        }
        bool fits = true;
        ix.list_ptr.assign(1, 0);
        fill(lo,
             [&](const Range& r, int e0, int n, int a, int b) { fits = put(ix.narrow, r, e0, n, chunks > 1 ? NARROW_ROWS : n * G, a, b) && fits; },
             [&]() { ix.list_ptr.push_back((int32_t)ix.narrow.size()); });
        if (!fits) return HARTS_EINVAL;
    }
    ix.n_parts = (int32_t)n_parts;
    ix.part_ptr.assign(1, 0);
    for (int32_t r = 0; r < n_q; r++) {
        if (parts[r].size() == 1) parts[r][0] = -1;               // written by its unit
        else ix.merged = 1;
        ix.part.insert(ix.part.end(), parts[r].begin(), parts[r].end());
        ix.part_ptr.push_back((int32_t)ix.part.size());
    }
    for (Entry& x : ix.entries)
        if (parts[x.row].size() == 1) x.most = -x.most - 1;
    return HARTS_OK;
}

}  // namespace

extern "C" int32_t harts_gen_attn_index(int32_t n_trees, const int32_t* tree_node_ptr, const int32_t* node_parent,
                                        const int32_t* node_fork_off, const int32_t* node_len, const int32_t* node_page_ptr,
                                        const int32_t* node_page, int32_t page, int32_t n_q, const int32_t* q_node, const int32_t* q_pos,
                                        int32_t Hq, int32_t Hkv, int32_t grow, int64_t cap_words, int32_t* blob, int64_t* n_words) {
    if (n_trees < 0 || n_q < 0 || grow < 0 || !tree_node_ptr || !node_page_ptr || !n_words || Hkv < 1 || Hq < Hkv || Hq % Hkv != 0 || Hq > 65535 || (int64_t)n_q * Hq > INT32_MAX ||
        (page != 16 && page != 32 && page != 64 && page != 128))
        return HARTS_EINVAL;
    if (tree_node_ptr[0] != 0 || node_page_ptr[0] != 0) return HARTS_EINVAL;
    if (n_trees > 0 && (!node_parent || !node_fork_off || !node_len)) return HARTS_EINVAL;
    if (n_q > 0 && (!q_node || !q_pos)) return HARTS_EINVAL;
    // ascending, before anything is read at their places: what lies between is then inside the arrays
    for (int32_t t = 0; t < n_trees; t++)
        if (tree_node_ptr[t + 1] <= tree_node_ptr[t]) return HARTS_EINVAL;
    for (int32_t v = 0; v < tree_node_ptr[n_trees]; v++)
        if (node_page_ptr[v + 1] < node_page_ptr[v]) return HARTS_EINVAL;
    try {
        if (!forest_ok(n_trees, tree_node_ptr, node_parent, node_fork_off, node_len)) return HARTS_EINVAL;
        if (node_page_ptr[tree_node_ptr[n_trees]] > 0 && !node_page) return HARTS_EINVAL;
        Index ix;
        const int32_t rc = build(n_trees, tree_node_ptr, node_parent, node_fork_off, node_len, node_page_ptr, node_page, page, n_q, q_node, q_pos, Hq, Hkv,
                                 grow, ix);
        if (rc != HARTS_OK) return rc;
        const int64_t n_pages = node_page_ptr[tree_node_ptr[n_trees]];
        int64_t total = HARTS_GEN_ATTN_HEADER_WORDS, at[7];
        const int64_t sizes[7] = {(int64_t)(ix.narrow.size() * sizeof(Unit) / 4), (int64_t)(ix.wide.size() * sizeof(Unit) / 4),
                                  (int64_t)(ix.entries.size() * sizeof(Entry) / 4), n_pages, n_q + 1, (int64_t)ix.part.size(), (int64_t)ix.list_ptr.size()};
        for (int i = 0; i < 7; i++) {
            at[i] = total;
            total += (sizes[i] + 3) & ~int64_t(3);            // 16-byte aligned starts
        }
        if (total >= INT32_MAX) return HARTS_EINVAL;
        *n_words = total;
        if (!blob) return HARTS_OK;
        if (cap_words < total) return HARTS_EINVAL;
        std::fill(blob, blob + total, 0);
        blob[N_Q] = n_q;
        blob[HQ] = Hq;
        blob[HKV] = Hkv;
        blob[PAGE] = page;
        blob[N_NARROW] = (int32_t)ix.narrow.size();
        blob[N_WIDE] = (int32_t)ix.wide.size();
        blob[N_PARTS] = ix.n_parts;
        blob[MERGED] = ix.merged;
        blob[MAX_PAGE] = ix.max_page;
        blob[WORDS] = (int32_t)total;
        for (const Unit& u : ix.narrow) blob[NARROW_MAX] = std::max(blob[NARROW_MAX], u.n);
        for (int i = 0; i < 6; i++) blob[NARROW + i] = (int32_t)at[i];
        blob[N_LISTS] = std::max<int32_t>(0, (int32_t)ix.list_ptr.size() - 1);
        blob[LIST_PTR] = (int32_t)at[6];
        auto put = [&](int i, const void* p, int64_t words) {
            if (words) std::copy_n(static_cast<const int32_t*>(p), words, blob + at[i]);
        };
        put(0, ix.narrow.data(), sizes[0]);
        put(1, ix.wide.data(), sizes[1]);
        put(2, ix.entries.data(), sizes[2]);
        put(3, node_page, sizes[3]);
        put(4, ix.part_ptr.data(), sizes[4]);
        put(5, ix.part.data(), sizes[5]);
        put(6, ix.list_ptr.data(), sizes[6]);
    } catch (const std::bad_alloc&) {
        return HARTS_ENOMEM;
    } catch (...) {
        return HARTS_EINTERNAL;
    }
    return HARTS_OK;
}
