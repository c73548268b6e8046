// Planner of attention for query blocks: the newest rows of a batch of sequences
// attend through sliding windows, sinks and drafted trees.  Plain C++17, no CUDA.
//
// Every sequence's queries are cut into blocks of up to kPrefillQTiles query
// tiles.  A block lists the 64-slot boxes in which some query of it sees a row,
// two to a key tile; each block is a unit at every KV head, and units are cut
// into items that give the CTAs even work.
#pragma once

#include <algorithm>
#include <cstring>
#include <functional>

#include "core.hpp"

namespace sq {

struct BlockPlanHost {
    std::vector<PrefillTile> tiles;
    std::vector<BlockItem> items;      // one: by CTA (see BlockItem::next); else longest first
    std::vector<BlockMerge> merges;    // units of more than one item
    std::vector<int32_t> tile_pages;   // [tiles][n_pieces] page of each piece, -1: none
    std::vector<int32_t> rows;         // [queries][2] first and last slot of each one's
                                       // window; empty: low0 + i, pos0 + i of the items
    std::vector<uint32_t> bits;        // [queries][n_words], drafted trees only
    int32_t n_words = 0, n_pieces = 0, BP = 0, n_parts = 0, max_splits = 0;
    int32_t n_ctas = 0;
    int32_t unit_rows = 0;             // rows of a tile pair that can hold queries
    bool one = true;                   // every item's queries fit in one query tile
};

// What the planner needs of one sequence of the call.
struct BlockSeq {
    const Seq* s;
    int32_t n_q;
    const int32_t* parents;  // null: no tree
};

namespace blocks_detail {

inline int32_t ceil_div(int64_t a, int64_t b) { return (int32_t)((a + b - 1) / b); }

// A sequence's rows as slots (page index x P + slot).
struct Slots {
    const Seq* s;
    int32_t P;
    bool partial;
    std::vector<int32_t> start;   // first row of each page (partial pages only)
    Slots(const Seq* seq, int32_t page_size) : s(seq), P(page_size), partial(has_partial_pages(*seq, P)) {
        if (!partial) return;
        start.assign(s->fill.size() + 1, 0);
        for (size_t q = 0; q < s->fill.size(); ++q) start[q + 1] = start[q] + s->fill[q];
    }
    int32_t of(int32_t row) const {
        if (!partial) return row;
        const int32_t q = (int32_t)(std::upper_bound(start.begin(), start.end(), row) - start.begin()) - 1;
        return q * P + (row - start[q]);
    }
    // Which of the 32 slots from k on (a multiple of 32) hold rows.
    uint32_t word(int32_t k, int32_t end) const {
        uint32_t w = 0;
        if (!partial) {
            const int32_t m = end - k;
            return m >= 32 ? 0xffffffffu : (m <= 0 ? 0u : (1u << m) - 1u);
        }
        for (int32_t i = 0; i < 32 && k + i < end; ++i)
            if ((k + i) % P < s->fill[(k + i) / P]) w |= 1u << i;
        return w;
    }
};

struct Unit {
    int32_t t0, T, q_row, n_q, n, pos0, low0, sink_end, base;
};

// A piece of a unit's key tiles.
struct Piece {
    int32_t unit, head, t0, n_tiles;
};

// Two-tile units are handed out item by item (longest first, to whichever CTA is
// free), so only their lengths matter: into how many pieces is each cut?  The
// estimate of a cut plays the hand-out through; an item costs its key tiles and a
// fixed part, and where units are cut at all the merge's launch comes on top.
inline void cut_units(const std::vector<Unit>& units, int32_t heads, int32_t ctas, int64_t max_parts,
                      std::vector<int32_t>* pieces) {
    // in key tiles.  Measured: 6 and 5 at D = 64 cut the five ragged chunks of 16/4
    // heads too little (17.8 us against 14.2), and moved no other shape by 1%
    constexpr double item = 3.0, merge = 2.5;
    pieces->assign(units.size(), 1);
    int32_t T_max = 0;
    int64_t total = 0;
    for (const Unit& u : units) {
        T_max = std::max(T_max, u.T);
        total += u.T;
    }
    // (many items each: they even out)
    if (T_max < 2 || (int64_t)units.size() * heads > 8 * (int64_t)ctas) return;
    double best = 0;
    int32_t best_len = T_max;
    static const int32_t cuts[] = {1, 2, 3, 4, 5, 6, 8, 11, 16, 24, 40, 64};
    std::vector<int32_t> count(T_max + 1);  // items of each length
    std::vector<double> load;
    for (int32_t k : cuts) {
        if (k > T_max) break;
        const int32_t len = ceil_div(T_max, k);
        std::fill(count.begin(), count.end(), 0);
        int64_t parts = 0, items = 0;
        for (const Unit& u : units) {
            const int32_t c = std::max(1, ceil_div(u.T, len));
            count[ceil_div(u.T, c)] += c * heads;
            items += (int64_t)c * heads;
            if (c > 1) parts += (int64_t)c * heads;
        }
        if (parts > max_parts || items > 16 * (int64_t)ctas) break;
        load.assign(ctas, 0.0);  // a heap, the least loaded CTA in front
        double most = 0;
        for (int32_t t = T_max; t > 0; --t)
            for (int32_t x = 0; x < count[t]; ++x) {
                std::pop_heap(load.begin(), load.end(), std::greater<double>());
                load.back() += t + item;
                most = std::max(most, load.back());
                std::push_heap(load.begin(), load.end(), std::greater<double>());
            }
        const double cost = most + (parts > 0 ? merge + 0.02 * parts : 0.0);
        if (k == 1 || cost < 0.97 * best) {
            best = cost;
            best_len = len;
        }
        if (cost > 1.3 * best) break;
    }
    for (size_t i = 0; i < units.size(); ++i)
        (*pieces)[i] = std::max(1, std::min(kPrefillMaxSplit, ceil_div(units[i].T, best_len)));
}

// One-tile units are bound by HBM, so every CTA gets an even share of the key
// tiles: the units' heads in a line, cut into stretches of equal cost (key tiles
// and a fixed part for each piece).  A cut is moved to a unit's end when it would
// leave a sliver on either side.  Short units are left whole while that leaves no
// CTA with a second one: a merge would cost more than it saves.  Without room for
// partial results no unit is cut: the longest first, each goes to the CTA that has
// least.
// pieces[c]: those of CTA c, in order.
inline void deal_units(const std::vector<Unit>& units, int32_t heads, int32_t ctas, int64_t max_parts,
                       int32_t D, std::vector<std::vector<Piece>>* out) {
    const double fixed = D == 128 ? 2.0 : 4.0;  // in key tiles
    const int32_t sliver = D == 128 ? 2 : 3, short_unit = D == 128 ? 6 : 12;
    out->clear();
    int64_t total = 0;
    int32_t T_max = 0;
    for (const Unit& u : units) {
        total += (int64_t)u.T * heads;
        T_max = std::max(T_max, u.T);
    }
    const int64_t n = (int64_t)units.size() * heads;
    const bool whole = max_parts < 2 || (n <= ctas && T_max <= short_unit);
    if (whole && n > ctas) {
        std::vector<int32_t> order(units.size());
        for (size_t u = 0; u < order.size(); ++u) order[u] = (int32_t)u;
        std::stable_sort(order.begin(), order.end(), [&](int32_t x, int32_t y) { return units[x].T > units[y].T; });
        typedef std::pair<double, int32_t> Load;  // and its CTA; the least in front
        std::vector<Load> load;
        for (int32_t c = 0; c < ctas; ++c) load.push_back({0.0, c});
        out->resize(ctas);
        for (int32_t u : order)
            for (int32_t h = 0; h < heads; ++h) {
                std::pop_heap(load.begin(), load.end(), std::greater<Load>());
                (*out)[load.back().second].push_back({u, h, 0, units[u].T});
                load.back().first += units[u].T + fixed;
                std::push_heap(load.begin(), load.end(), std::greater<Load>());
            }
        return;
    }
    // (a cut at the end of each share adds a piece)
    // and a unit has at most kPrefillMaxSplit pieces
    const double share = std::max({2.0 * sliver, (total + fixed * n) / ctas + fixed,
                                   (double)T_max / (kPrefillMaxSplit - 1) + fixed});
    out->emplace_back();
    double room = share;  // what the last CTA may still take; the next begins with the rest

    int64_t parts = 0;
    for (int32_t u = 0; u < (int32_t)units.size(); ++u)
        for (int32_t h = 0; h < heads; ++h) {
            const int32_t T = units[u].T;
            int32_t at = 0, cut = 0;  // tiles dealt, pieces so far
            while (at < T) {
                const int32_t left = T - at;
                int32_t take = left;
                const bool may = (int32_t)out->size() < ctas;
                if (whole) {
                    if (may && !out->back().empty()) {
                        out->emplace_back();
                        room += share;
                    }
                } else if (may && left + fixed > room + sliver) {
                    take = (int32_t)(room - fixed);
                    // too little room for a piece worth its start
                    if (take < sliver) {
                        if (!out->back().empty()) {
                            out->emplace_back();
                            room += share;
                            continue;
                        }
                        take = std::min(left, sliver);
                    }
                    if (left - take < sliver || cut + 1 >= kPrefillMaxSplit || parts + 2 > max_parts) take = left;
                }
                if (take < left || cut > 0) ++parts;
                out->back().push_back({u, h, at, take});
                room -= take + fixed;
                at += take;
                ++cut;
                if (!whole && may && room < sliver + fixed) {
                    out->emplace_back();
                    room += share;
                }
            }
        }
    if (out->back().empty()) out->pop_back();
}

}  // namespace blocks_detail

// Plans one call (kPrefillPartLimit bytes of partial results, or `part_limit`).
// The arguments have been checked but for the drafted rows' slots (kUnsupported)
// and the plan's size (kCapacity).  A call whose sequences have at most `most_one` query
// tiles each is planned a tile at a time, others by pairs of tiles.
inline int plan_blocks(const Geometry& g, const std::vector<BlockSeq>& seqs, int32_t window, int32_t n_sink,
                       int32_t ctas, int64_t part_limit, BlockPlanHost* out, int32_t most_one = 1) {
    using namespace blocks_detail;
    *out = BlockPlanHost();
    const int32_t P = g.P, BP = kPrefillRows / g.G();
    out->BP = BP;
    const int32_t br = std::min(P, 64), half = 64 / br;
    out->n_pieces = 2 * half;
    bool table = false;
    int64_t queries = 0;
    for (const BlockSeq& q : seqs) {
        queries += q.n_q;
        if (q.n_q > (int64_t)BP * most_one) out->one = false;
        if (q.n_q > 0) table |= q.parents || has_partial_pages(*q.s, P);
    }
    if (queries > 0x7fffffff / std::max(1, g.Hq)) return kCapacity;
    if (table) out->rows.resize(2 * (size_t)queries);
    // words of a drafted row's bitmap: the tree may begin anywhere in its first
    for (const BlockSeq& q : seqs)
        if (q.parents && q.n_q > 0) out->n_words = std::max(out->n_words, (q.n_q + 31) / 32 + 1);
    if (out->n_words) out->bits.assign((size_t)queries * out->n_words, 0);
    std::vector<Unit> units;
    int32_t q_row = 0;
    for (const BlockSeq& q : seqs) {
        const int32_t m = q.n_q;
        if (m == 0) continue;
        const Seq& s = *q.s;
        const Slots at(&s, P);
        const int32_t end = slot_end(s, P), ctx = s.n - m;
        const int32_t reach = window > 0 ? std::min(window, s.n + 1) : s.n + 1;
        int32_t base = kBlockNoTree;
        std::vector<int32_t> depth, low(m), top(m);
        const int32_t sinks = q.parents ? std::min(n_sink, ctx) : std::min(n_sink, s.n);
        const int32_t sink_end = sinks > 0 ? at.of(sinks - 1) + 1 : 0;
        if (q.parents) {
            const int32_t d0 = at.of(ctx);
            if (at.of(s.n - 1) - d0 != m - 1) return kUnsupported;
            base = d0 / 32 * 32;
            // the ancestors of each drafted row, itself among them
            const int32_t w = (m + 31) / 32;
            std::vector<uint32_t> anc((size_t)m * w, 0);
            depth.assign(m, 0);
            for (int32_t i = 0; i < m; ++i) {
                const int32_t p = q.parents[i];
                if (p >= 0) {
                    depth[i] = depth[p] + 1;
                    std::copy_n(&anc[(size_t)p * w], w, &anc[(size_t)i * w]);
                }
                anc[(size_t)i * w + i / 32] |= 1u << (i % 32);
                const int64_t pos = (int64_t)ctx + depth[i];
                const int32_t first = (int32_t)std::max<int64_t>(0, pos - reach + 1);
                low[i] = at.of(std::min(first, ctx));
                top[i] = base - 1;
                uint32_t* row = &out->bits[(size_t)(q_row + i) * out->n_words];
                // context rows that share the tree's first word
                for (int32_t k = base; k < d0; ++k)
                    if (k >= low[i] || k < sink_end) row[0] |= 1u << (k - base);
                for (int32_t j = 0; j <= i; ++j) {
                    if (!((anc[(size_t)i * w + j / 32] >> (j % 32)) & 1u)) continue;
                    const int64_t pj = (int64_t)ctx + depth[j];
                    if (pj <= pos - reach && pj >= n_sink) continue;
                    row[(d0 + j - base) / 32] |= 1u << ((d0 + j - base) % 32);
                }
            }
        } else {
            for (int32_t i = 0; i < m; ++i) {
                const int32_t p = ctx + i;
                // (slots are rows unless pages are partial)
                low[i] = at.partial ? at.of(std::max(0, p - reach + 1)) : p - reach + 1;
                top[i] = at.of(p);
            }
        }
        if (table)
            for (int32_t i = 0; i < m; ++i) {
                out->rows[2 * (size_t)(q_row + i)] = low[i];
                out->rows[2 * (size_t)(q_row + i) + 1] = top[i];
            }
        const int32_t span = out->one || m <= BP ? BP : BP * kPrefillQTiles;
        out->unit_rows =
            std::max(out->unit_rows, span == BP ? std::min(m, BP) * g.G() : kPrefillQTiles * kPrefillRows);
        for (int32_t b = 0; b < m; b += span) {
            const int32_t e = std::min(m, b + span);
            int32_t lo = 0x7fffffff, hi = 0;
            for (int32_t i = b; i < e; ++i) lo = std::min(lo, std::max(0, low[i]));
            hi = q.parents ? at.of(ctx + e - 1) : top[e - 1];
            // boxes of the sinks before the window's, then the window's
            const int32_t lo_box = lo / 64, hi_box = hi / 64;
            const int32_t sink_boxes = std::min(lo_box, ceil_div(std::min(sink_end, hi + 1), 64));
            Unit u;
            u.t0 = (int32_t)out->tiles.size();
            u.q_row = q_row + b;
            u.n_q = e - b;
            u.n = end;
            u.pos0 = top[b];
            u.low0 = low[b];
            u.sink_end = sink_end;
            u.base = base;
            bool upper = false;
            auto add = [&](int32_t box) {
                const int32_t k = box * 64;
                const uint32_t w0 = at.word(k, end), w1 = at.word(k + 32, end);
                if (!(w0 | w1)) return;
                if (!upper) {
                    out->tiles.push_back(PrefillTile{});
                    out->tile_pages.resize(out->tile_pages.size() + out->n_pieces, -1);
                    out->tiles.back().key0b = kPrefillNoKeys;
                }
                PrefillTile& t = out->tiles.back();
                (upper ? t.key0b : t.key0) = k;
                t.vis[upper ? 2 : 0] = w0;
                t.vis[upper ? 3 : 1] = w1;
                if (upper && (t.vis[0] & t.vis[1] & w0 & w1) == 0xffffffffu) t.flags = kPrefillTileFull;
                int32_t* pg = &out->tile_pages[out->tile_pages.size() - out->n_pieces + (upper ? half : 0)];
                for (int32_t i = 0; i < half; ++i)
                    if (k + i * br < end) pg[i] = s.pages[(k + i * br) / P];
                upper = !upper;
            };
            for (int32_t x = 0; x < sink_boxes; ++x) add(x);
            for (int32_t x = lo_box; x <= hi_box; ++x) add(x);
            u.T = (int32_t)out->tiles.size() - u.t0;
            if ((int64_t)out->tiles.size() > kMaxBlockTiles) return kCapacity;
            units.push_back(u);
        }
        q_row += m;
    }
    const int64_t max_parts = part_limit / prefill_part_bytes(g.D);
    auto item_of = [&](const Piece& p, int32_t part) {
        const Unit& u = units[p.unit];
        return BlockItem{p.head | (u.n_q > BP ? kBlockTwoTiles : 0), u.t0 + p.t0, p.n_tiles, part, u.q_row, u.n_q,
                         u.n, u.pos0, u.low0, u.sink_end, u.base, -1};
    };
    if (out->one) {
        std::vector<std::vector<Piece>> dealt;
        deal_units(units, g.Hkv, std::max(1, ctas), max_parts, g.D, &dealt);
        // pieces of a unit follow one another over the CTAs: number them as they come
        out->n_ctas = (int32_t)dealt.size();
        std::vector<BlockItem> rest;
        out->items.reserve(dealt.size());
        for (size_t c = 0; c < dealt.size(); ++c)
            for (size_t x = 0; x < dealt[c].size(); ++x) {
                const Piece& p = dealt[c][x];
                int32_t part = -1;
                if (p.n_tiles < units[p.unit].T) {
                    if (p.t0 == 0)
                        out->merges.push_back({p.head, out->n_parts, 0, units[p.unit].q_row, units[p.unit].n_q,
                                               {0, 0, 0}});
                    out->max_splits = std::max(out->max_splits, ++out->merges.back().n);
                    part = out->n_parts++;
                }
                BlockItem it = item_of(p, part);
                if (x + 1 < dealt[c].size())  // (its place once the first ones are in)
                    it.next = (int32_t)(dealt.size() + rest.size()) + (x == 0 ? 0 : 1);
                if (x == 0) out->items.push_back(it);
                else rest.push_back(it);
            }
        out->items.insert(out->items.end(), rest.begin(), rest.end());
        return kOk;
    }
    std::vector<int32_t> pieces;
    cut_units(units, g.Hkv, std::max(1, ctas), max_parts, &pieces);
    // items, longest first; the heads of one block side by side (their queries and
    // pages are neighbours)
    std::vector<std::pair<int32_t, int32_t>> order;  // (longest piece, unit)
    order.reserve(units.size());
    size_t n_items = 0;
    for (size_t i = 0; i < units.size(); ++i) {
        order.push_back({ceil_div(units[i].T, pieces[i]), (int32_t)i});
        n_items += (size_t)pieces[i] * g.Hkv;
    }
    std::stable_sort(order.begin(), order.end(),
                     [](const std::pair<int32_t, int32_t>& a, const std::pair<int32_t, int32_t>& b) {
                         return a.first > b.first;
                     });
    out->items.reserve(n_items);
    for (const auto& o : order) {
        const Unit& u = units[o.second];
        const int32_t k = pieces[o.second], part0 = out->n_parts;
        if (k > 1) {
            for (int32_t h = 0; h < g.Hkv; ++h)
                out->merges.push_back({h, part0 + h * k, k, u.q_row, u.n_q, {0, 0, 0}});
            out->n_parts += k * g.Hkv;
            out->max_splits = std::max(out->max_splits, k);
        }
        for (int32_t x = 0; x < k; ++x)
            for (int32_t h = 0; h < g.Hkv; ++h) {
                const int32_t a = (int32_t)((int64_t)u.T * x / k), b = (int32_t)((int64_t)u.T * (x + 1) / k);
                out->items.push_back(item_of({o.second, h, a, b - a}, k > 1 ? part0 + h * k + x : -1));
            }
    }
    out->n_ctas = (int32_t)out->items.size();
    return kOk;
}

}  // namespace sq
