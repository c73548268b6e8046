// The planner of attention for query blocks, for CPU tests (part of
// libsq_host.so; see host_test_api.cpp).
#include <cstring>

#include "../host/blocks.hpp"

using namespace sq;

extern "C" {

// Plans a call over the sequences of a host cache.  info: tiles, items, merges,
// rows (0 or queries), n_words, n_pieces, BP, n_parts, one, unit_rows,
// max_splits, n_ctas.  Arrays of the plan are copied to the non-null buffers (which the
// caller sizes by a first call without them).
int sqh_plan_blocks(void* c, const int32_t* handles, int32_t n_seqs, const int32_t* n_q,
                    const int32_t* parents, int32_t window, int32_t n_sink, int32_t ctas,
                    int64_t part_limit, int64_t* info, int32_t* tiles, int32_t* items, int32_t* merges,
                    int32_t* rows, uint32_t* bits, int32_t* tile_pages) {
    HostCache* h = static_cast<HostCache*>(c);
    std::vector<BlockSeq> seqs;
    for (int32_t i = 0, at = 0; i < n_seqs; at += n_q[i++])
        seqs.push_back({h->seq(handles[i]), n_q[i], parents ? parents + at : nullptr});
    BlockPlanHost p;
    const int rc = plan_blocks(h->geom(), seqs, window, n_sink, ctas, part_limit, &p);
    if (rc != kOk) return rc;
    const int64_t v[] = {(int64_t)p.tiles.size(), (int64_t)p.items.size(), (int64_t)p.merges.size(),
                         (int64_t)p.rows.size() / 2, p.n_words, p.n_pieces, p.BP, p.n_parts, p.one,
                         p.unit_rows, p.max_splits, p.n_ctas};
    std::memcpy(info, v, sizeof v);
    auto put = [](void* to, const void* from, size_t n) {
        if (to && n) std::memcpy(to, from, n);
    };
    put(tiles, p.tiles.data(), p.tiles.size() * sizeof(PrefillTile));
    put(items, p.items.data(), p.items.size() * sizeof(BlockItem));
    put(merges, p.merges.data(), p.merges.size() * sizeof(BlockMerge));
    put(rows, p.rows.data(), p.rows.size() * 4);
    put(bits, p.bits.data(), p.bits.size() * 4);
    put(tile_pages, p.tile_pages.data(), p.tile_pages.size() * 4);
    return kOk;
}

// Plans windowed decode; layout and buffer as sqh_plan_decode's.
int sqh_plan_window_decode(void* c, const int32_t* handles, int32_t n_seqs, int32_t n_ctas,
                           int32_t window, int32_t n_sink, int64_t* layout_out, uint8_t* buf,
                           int64_t buf_bytes) {
    HostCache* h = static_cast<HostCache*>(c);
    DecodePlanHost p;
    const int rc = plan_window_decode(*h, handles, n_seqs, n_ctas, window, n_sink, &p);
    if (rc != kOk) return rc;
    const DecodePlanLayout L = plan_layout(p, n_seqs, h->geom().Hkv);
    const int64_t v[] = {L.segs, L.items, L.cta_begin, L.page_ids, L.comb_off, L.arrive, L.total,
                         L.n_segs, L.n_items, L.n_ctas, L.n_page_ids, L.n_comb_keys, L.n_comb_ent,
                         p.unique_tokens, p.logical_tokens, (int64_t)sizeof(DecodeSeg), L.page_fill};
    std::memcpy(layout_out, v, sizeof v);
    if (buf) {
        if (buf_bytes < L.total) return kInvalidArg;
        plan_serialize(p, L, buf);
    }
    return kOk;
}

}  // extern "C"
