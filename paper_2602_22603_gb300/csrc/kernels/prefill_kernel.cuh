// Masked prefill attention on the 5th-generation tensor cores.
//
// What it computes (Algorithm 2, BuildMask; Sec. 3.3): the last n_q tokens of
// a sequence attend causally to its tokens, with the tokens of the given spans
// (closed cursors) removed from every query's view:
//   query at position p, query head h, KV head g = floor(h / G):
//     s_j = sm_scale * q_h . k_{g,j}   for visible keys j (j <= p, j in no span)
//     o_h = sum_j softmax_j(s) v_{g,j}
//
// A query tile is 128 rows: floor(128 / G) consecutive query positions times
// the G query heads of one KV head (Sec. 2.1).  One CTA owns two consecutive
// query tiles (a, b) of the same KV head, and every K/V tile it loads serves
// both, which halves the loads per tensor-core FLOP.  Keys go 128 at a time;
// tiles whose keys are all masked are never loaded (the host lists the others
// with a visibility bitmap).  Per key tile j and query tile t:
//   S_t = Q_t K_j^T           tcgen05.mma, Q and K from shared memory, S in TMEM
//   P_t = exp2(S_t - m)       softmax warpgroup t: tcgen05.ld of S, mask, bf16 P
//                             stored back over the first half of S_t
//   O_t += P_t V_j            tcgen05.mma with A = P from TMEM and V read
//                             token-major from shared memory (MN-major B)
// The MMA issuer interleaves the two tiles (PV_a(j), S_a(j+1), PV_b(j),
// S_b(j+1)), so while one warpgroup turns S into P the tensor core works for
// the other.  P_t(j) shares TMEM with S_t: S_t(j+1) is issued after PV_t(j),
// and tcgen05.mma operations of one thread execute in issue order.  The same
// order means that when S_t(j) is ready, PV_t(j-1) is complete, so a
// warpgroup may rescale O_t then without another wait.  The running maximum
// is raised lazily: a key tile's weights are taken with the current maximum
// and accepted while every row's sum of them stays at most 2^16 (so does each
// weight; 2^8 in warps with rows that are no query); only then is a maximum
// raised and O rescaled.  K and V stream through
// one ring of shared-memory slots (K_0, V_0, K_1, ...); V_j and K_{j+1} are
// released together, after the products PV_b(j) and S_b(j+1).
//
// What bounds it: the one thread that issues the MMAs (see there), then the
// softmax chain of each tile.  32,768 queries, 40% masked, 32q/8kv, d = 128:
// 3.55 -> 3.25 ms a layer (1,320 -> 1,440 TFLOP/s
// over the visible pairs); 3,001 queries over 33,001 tokens: 1,027 -> 845 us.
//
// Short query blocks: when a CTA tile's queries all fit in tile a, tile b's
// warpgroup takes the same rows over every other key tile (dual-key mode, the
// two results merged per row at the end, loads in the order the MMAs consume
// them).
//
// Work items: the host lists (CTA tile, KV head, key range) items, longest
// first, and the grid has one CTA per item, of which an SM holds one.  A CTA
// that has issued most loads of its item asks the launch hardware for the next
// CTA not started yet (clusterlaunchcontrol.try_cancel) and takes over its
// item, so the ring, the barriers' phases and tensor memory run on from item
// to item and the next item's first keys and queries load while the last one's
// softmax, PV and output finish.  One CTA per item paid a start and a drain
// each, ~5 us; dealing the items to persistent CTAs beforehand lost 4%, since
// SMs run this kernel at speeds up to 7% apart (1.78 to 1.91 us per key tile).
// A unit split in several items (too few units for the SMs, or a last round
// that would leave most SMs idle) leaves normalised partial results that a
// second kernel merges.
//
// Calls whose queries fit in one query tile (kOneTile: the 8-query calls of an
// auxiliary thread, every item dual-key) run an instance without the two-tile
// path.  HBM bounds them, so, when the plan was on the device before, their
// producer loads its item's first two key tiles before the dependency wait,
// while the previous launch's last CTAs finish and are merged: 8 queries over
// 131,080 tokens, 87.0 -> 85.4 us a layer (79 at the read probe's rate).  Loading early in the two-tile instance gained nothing (the
// issuing lane bounds it) and lost 1 to 2% to the code generated around it; a
// ring one slot longer (the second query tile's space), or L2 prefetches beyond
// the ring, slow the CTAs still at work by more than they save the next ones.
//
// Query blocks (kBlocks): the same kernel for the newest tokens of a batch of
// sequences, with windows, sinks and drafted trees.  An item carries its own
// sequence's end, its first query's row and the rule of its mask, and every block
// of queries has a list of its own of the 64-key boxes that some query of it
// sees; the roles, the ring and the products are those above.
//
// Warp roles (320 threads): warp 0 loads (lanes 0 and 1 issue the TMA copies,
// two loads at a time; query blocks: a lane to a box), lane 0 of warp 1 issues
// the MMAs and warp 1 owns the TMEM allocation, warps 2-5
// are the softmax warpgroup of tile a and warps 6-9 that of tile b (warp w
// reads TMEM lanes 32 (w mod 4) .. +31, one row per thread), and warp 10, in
// instances that have it, is the second producer.  Every wait is
// bounded; a wait that runs out sets the error word and the CTA winds down
// after its copies and MMAs in flight have completed.
#pragma once

#include <type_traits>

#include "e4m3.cuh"
#include "operators.hpp"
#include "ptx.cuh"
#include "tc.cuh"

namespace sq {
namespace dev {
namespace {

// Instances.  kOneTile: every query of an item fits in tile a.  kBlocks: items
// carry what they need of their own sequence and have key tiles of their own
// (query blocks of a batch, see BlockItem); otherwise all items belong to one
// sequence, whose newest n_q tokens they share out.  kTwoProducers: blocks whose loads
// are two producer warps': on pages of fewer than 64 tokens, which take many boxes,
// and one-tile blocks of 64 dimensions, whose loads are short.  kHides: prefill of a
// sequence whose hidden rows may hold anything (zero_hidden_values).
// kE8: rows in 8 bits (convert_tiles).
constexpr int kOneTile = 1, kBlocks = 2, kTwoProducers = 4, kHides = 8, kE8 = 16;
template <int M>
constexpr bool one_tile = (M & kOneTile) != 0;
template <int M>
constexpr bool of_blocks = (M & kBlocks) != 0;
template <int M>
constexpr bool hides = (M & kHides) != 0;
template <int M>
constexpr int producers = (M & kTwoProducers) != 0 ? 2 : 1;
template <int M>
constexpr bool e8 = (M & kE8) != 0;

// S buffers: one for each softmax warpgroup, and a third for one-tile blocks of 64
// dimensions, whose O leaves the columns (S_2 after O_b).  With two a warpgroup that has handed over
// P waits for its PV and for the QK after it before it has work again; with three that
// QK is done by then.  8 trees of 16 over 32,768 tokens, 64/8/64 heads, pages of 32:
// 121 -> 107 us by an issuing lane that waits for P alone, 100 with the third buffer.
template <int D, int M>
constexpr int s_buffers = D == 64 && (M & ~kE8) == (kBlocks | kOneTile | kTwoProducers) ? 3 : 2;

// Items in flight between the producer and the other roles, and the warps that
// read each (MMA warp and eight softmax warps).
constexpr int kItemSlots = 4;
constexpr int kItemReaders = 9;
// Warps that widen tiles (kE8): two groups that take alternate tiles, a warp to 32 rows.
constexpr int kConvertGroups = 2, kConverters = 4 * kConvertGroups;
constexpr int kProducer2 = 10;  // query blocks: the warp of their odd loads

template <int D, int M>
struct PreCfg {
    static constexpr int kThreads = e8<M> ? 640 : 320 + 32 * (producers<M> - 1);
    static constexpr int kColBlocks = D / 64;                  // 64-column (128-byte) blocks
    static constexpr int kBlockBytes = kPrefillRows * 128;      // one block of a 128-row tile
    static constexpr int kQBytes = kColBlocks * kBlockBytes;    // one query tile
    static constexpr int kSlotBytes = kColBlocks * kBlockBytes;  // 128 keys of K or of V
    static constexpr int kSlots = e8<M> ? (D == 128 ? 6 : 8) : (D == 128 ? 5 : 12);
    // (8 bits) where a tile's codes land: rows of 128 in the second half of its slot,
    // where the converter of a row writes what it has read; of 64 in space of their own
    static constexpr int kCodeStride = D == 128 ? kSlotBytes : kPrefillKeys * D;
    static constexpr int kTileScales = e8<M> ? kPrefillKeys / kScaleRows : 0;
    static constexpr int kOffQ = 0;
    static constexpr int kOffRing = kOffQ + (one_tile<M> ? 1 : kPrefillQTiles) * kQBytes;
    static constexpr int kOffCodes = kOffRing + (D == 128 ? kBlockBytes : kSlots * kSlotBytes);
    static constexpr int kOffBar = kOffRing + kSlots * (kSlotBytes + (e8<M> && D == 64 ? kCodeStride : 0));
    static constexpr int kBarQ = 0;
    static constexpr int kBarFull = 1;                  // [kSlots] tile landed (V: and ready)
    static constexpr int kBarEmpty = kBarFull + kSlots; // [kSlots] slot consumed by the MMAs
    static constexpr int kBarS = kBarEmpty + kSlots;    // [2] S_t written (and PV_t before it done)
    static constexpr int kBufs = s_buffers<D, M>;
    static constexpr int kBarP = kBarS + kBufs;         // [2] P_t written (128 arrivals)
    static constexpr int kBarO = kBarP + kBufs;         // [2] last PV_t done
    static constexpr int kBarPV = kBarO + 2;            // (three S buffers) the last PV but two done
    static constexpr int kBarVfix = kBarPV + (kBufs > 2 ? 1 : 0);          // V of the last key tile landed
    static constexpr int kBarQFree = kBarVfix + 1;      // the item's last QK product done
    static constexpr int kBarDone = kBarQFree + 1;      // every MMA of the CTA done
    static constexpr int kBarItem = kBarDone + 1;       // [kItemSlots] item written
    static constexpr int kBarItemFree = kBarItem + kItemSlots;  // [kItemSlots] item read by all
    static constexpr int kBarClc = kBarItemFree + kItemSlots;   // answer of the launch hardware
    static constexpr int kBarX = kBarClc + 1;           // dual-key mode: tile b's half handed over
    static constexpr int kBarXFree = kBarX + 1;         // ... and read by tile a
    static constexpr int kBarRaw = kBarXFree + 1;       // (8 bits) [kSlots] codes and scales landed
    static constexpr int kNumBars = kBarRaw + (e8<M> ? kSlots : 0);
    static constexpr int kItemBytes = of_blocks<M> ? (int)sizeof(BlockItem) : (int)sizeof(PrefillItem);
    static constexpr int kOffItems = (kOffBar + kNumBars * 8 + 15) & ~15;  // [kItemSlots] items
    static constexpr int kOffClc = kOffItems + kItemSlots * kItemBytes;   // 16-byte answer
    static constexpr int kOffMisc = kOffClc + 16;
    // dual-key mode: tile b's (max, normaliser) of each row, for the merge
    static constexpr int kOffXchg = (kOffMisc + 32 + 15) & ~15;
    // (8 bits) each slot's scales, and the rows of its tile that are the sequence's
    static constexpr int kOffScales = kOffXchg + kPrefillRows * 8;
    static constexpr int kOffRows = kOffScales + kSlots * kTileScales * 4;
    static constexpr int kSmemBytes = kOffRows + (e8<M> ? kSlots * 4 : 0) + 1024;  // + alignment slack
    // registers of a thread (8 bits; see the kernel): softmax warps, converters, others
    static constexpr int kSoftmaxRegs = 144, kConvertRegs = 56, kOtherRegs = 80;
    static constexpr int kAllRegs = 256 * kSoftmaxRegs + 32 * kConverters * kConvertRegs + 128 * kOtherRegs;
    static_assert(!e8<M> || kThreads * 96 >= kAllRegs, "register split");
    static constexpr uint32_t kTmemCols = 512;
    static constexpr uint32_t kColS = 0;    // S_t (fp32) at 128 t; P_t (bf16 pairs) over its first 64
    static constexpr uint32_t kColO = 256;  // O_t (fp32) at 256 + 128 t
    static constexpr uint32_t kOStep = kBufs > 2 ? 64 : 128;  // (256 + 64 t; S_2 at 384)
    __device__ static uint32_t col_s(uint32_t buf) {
        return kBufs > 2 && buf == 2 ? 384u : kColS + buf * kPrefillKeys;
    }
    static constexpr uint32_t kIdescQK = mma_idesc_bf16(128, kPrefillKeys, false);
    static constexpr uint32_t kIdescPV = mma_idesc_bf16(128, D, true);
    static_assert(kSmemBytes <= 232448, "shared memory");
    static_assert(kOffXchg % 16 == 0 && kOffRing % 1024 == 0 && kOffBar % 8 == 0, "alignment");
    static_assert(kPrefillQTiles == 2, "two query tiles per CTA");
};

struct Smem {
    uint32_t base;  // shared address of the 1024-aligned region
    uint8_t* ptr;
    template <int D, int M>
    __device__ uint32_t bar(int i) const {
        return base + PreCfg<D, M>::kOffBar + 8 * i;
    }
};

// A work item as the roles see it; raw.z (its key tiles) is -1 after the last.
struct Item {
    int g, pos_lo, t0, T, part;
    bool two;   // tile b holds query rows
    bool dual;  // tile b takes every other key tile of tile a's rows
};

template <int M>
__device__ __forceinline__ Item make_item(const PrefillArgs& a, int4 raw) {
    Item it;
    it.t0 = raw.y;
    it.T = raw.z;
    it.part = raw.w;
    // tile b is empty when every query of the CTA tile fits in tile a
    if constexpr (of_blocks<M>) {
        it.g = raw.x & (kBlockTwoTiles - 1);
        it.pos_lo = 0;
        it.two = !one_tile<M> && (raw.x & kBlockTwoTiles);
    } else {
        const int qt = raw.x / a.Hkv;
        it.g = raw.x - qt * a.Hkv;
        it.pos_lo = qt * kPrefillQTiles * a.BP;
        it.two = !one_tile<M> && it.pos_lo + a.BP < a.n_q;
    }
    it.dual = !it.two && it.T >= 2;
    return it;
}

// Asks the launch hardware for a CTA of the grid that has not started; the
// 16-byte answer lands at `dst`, completing `bar`.
__device__ __forceinline__ void clc_request(uint32_t dst, uint32_t bar) {
    asm volatile(
        "clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], "
        "[%1];" ::"r"(dst),
        "r"(bar)
        : "memory");
}

// The answer at `src`: the index of the CTA taken over, or -1.
__device__ __forceinline__ int clc_answer(uint32_t src) {
    uint32_t ok, x;
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b128 r;\n\t"
        "ld.shared.b128 r, [%2];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t"
        "mov.u32 %1, 0;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n\t}"
        : "=r"(ok), "=r"(x)
        : "r"(src)
        : "memory");
    return ok ? (int)x : -1;
}

// The reading side of the item ring: item k of the CTA is in slot k mod
// kItemSlots until every reader has freed it.
template <int D, int M>
__device__ __forceinline__ bool item_wait(const Smem& sm, uint32_t k, const volatile int* abort_flag) {
    return mbar_wait(sm.bar<D, M>(PreCfg<D, M>::kBarItem + k % kItemSlots),
                     (k / kItemSlots) & 1, abort_flag);
}
template <int D, int M>
__device__ __forceinline__ int4 item_read(const Smem& sm, uint32_t k) {
    using C = PreCfg<D, M>;
    return *reinterpret_cast<const int4*>(sm.ptr + C::kOffItems + k % kItemSlots * C::kItemBytes);
}
// ... what a block item has of its own sequence.
template <int D, int M>
__device__ __forceinline__ const BlockItem& item_block(const Smem& sm, uint32_t k) {
    using C = PreCfg<D, M>;
    static_assert(of_blocks<M>, "a block item");
    return *reinterpret_cast<const BlockItem*>(sm.ptr + C::kOffItems + k % kItemSlots * C::kItemBytes);
}
template <int D, int M>
__device__ __forceinline__ void item_free(const Smem& sm, uint32_t k) {
    mbar_arrive(sm.bar<D, M>(PreCfg<D, M>::kBarItemFree + k % kItemSlots));
}

// Bits 0 .. x of a word (x < 0: none; x >= 31: all).
__device__ __forceinline__ uint32_t low_bits_through(int x) {
    return x >= 31 ? 0xffffffffu : (x < 0 ? 0u : ((2u << x) - 1u));
}

// Order of the K and V loads of a CTA's T key tiles, load u into ring slot
// u mod kSlots.  Normally key tile by key tile: u = 2 j is K_j, u = 2 j + 1
// is V_j.  In dual-key mode (tile a takes the even key tiles, tile b the odd
// ones) the loads follow the order in which the MMA warp consumes them, so
// that no tile waits in the ring for a later one: K_0, K_1, then V_j and
// K_{j+2} in turn, and the last two V tiles.  (kLead: the K tiles ahead of their V,
// one for each S buffer.)
template <int kLead = 2>
__device__ __forceinline__ void load_of(int u, int T, bool dual, int& j, int& kv) {
    if (!dual) {
        j = u >> 1;
        kv = u & 1;
    } else if (u < kLead && (kLead == 2 || u < T)) {
        j = u;
        kv = 0;
    } else if (u >= 2 * T - kLead) {
        j = u - T;
        kv = 1;
    } else {
        const bool k = (u ^ kLead) & 1;
        j = ((u - kLead) >> 1) + (k ? kLead : 0);
        kv = k ? 0 : 1;
    }
}

// {first key of each half, page of box 0, page of box 1} of key tile
// tb + lane % kBatch of an item (x = key0, y = page 0, z = page 1, w = key0b).
constexpr int kBatch = 16;
__device__ __forceinline__ int4 tile_record(const PrefillArgs& a, int t0, int T, int tb, int lane) {
    int4 r = make_int4(0, -1, -1, kPrefillNoKeys);
    const int jj = tb + (lane & (kBatch - 1));
    if (jj < T) {
        const size_t t = (size_t)(t0 + jj);
        r.x = __ldg(&a.tiles[t].key0);
        r.w = __ldg(&a.tiles[t].key0b);
        r.y = __ldg(&a.tile_pages[t * a.n_pieces]);
        if (a.n_pieces > 1) r.z = __ldg(&a.tile_pages[t * a.n_pieces + 1]);
    }
    return r;
}

// Block items: what a lane needs of the piece that it loads in a batch of loads.  A
// load is n_pieces boxes of min(P, 64) rows, so 32 / n_pieces loads are a batch, a
// lane to a box; the batch's records are read together, a batch ahead of their use.
template <int M>
__device__ __forceinline__ int pieces_of(const PrefillArgs& a) { return producers<M> > 1 ? a.n_pieces : 2; }
template <int D, int M>
struct BlockBatch {
    int32_t key, page;  // the box's first key; its page, -1: no such box
    // the producer warp w's loads from its x0-th on
    __device__ __forceinline__ void read(const PrefillArgs& a, const Item& it, int x0, int w, int lane) {
        const int per = pieces_of<M>(a), i = lane & (per - 1), u = (x0 + lane / per) * producers<M> + w;
        key = 0;
        page = -1;
        if (u >= 2 * it.T) return;
        int j, kv;
        load_of<s_buffers<D, M>>(u, it.T, it.dual, j, kv);
        const PrefillTile* t = a.tiles + it.t0 + j;
        const int half = per >> 1, br = 64 / half;
        key = i < half ? __ldg(&t->key0) + i * br : __ldg(&t->key0b) + (i - half) * br;
        page = __ldg(&a.tile_pages[(size_t)(it.t0 + j) * per + i]);
    }
};

// The producer's copy of an item.
template <int M>
struct ItemRecord {
    int4 raw;
    int4 more[of_blocks<M> ? 2 : 1];  // (block items: q_row .. pos0, low0 ..)
    __device__ __forceinline__ void read(const PrefillArgs& a, int i) {
        if constexpr (of_blocks<M>) {
            const int4* p = reinterpret_cast<const int4*>(a.items) + 3 * (size_t)i;
            raw = __ldg(p);
            more[0] = __ldg(p + 1);
            more[1] = __ldg(p + 2);
        } else {
            raw = __ldg(reinterpret_cast<const int4*>(a.items) + i);
        }
    }
    __device__ __forceinline__ void copy(const uint8_t* slot) {
        const int4* p = reinterpret_cast<const int4*>(slot);
        raw = p[0];
        if constexpr (of_blocks<M>) {
            more[0] = p[1];
            more[1] = p[2];
        }
    }
    __device__ __forceinline__ void write(uint8_t* slot) const {
        int4* p = reinterpret_cast<int4*>(slot);
        p[0] = raw;
        if constexpr (of_blocks<M>) {
            p[1] = more[0];
            p[2] = more[1];
        }
    }
    // (block items) the CTA's next item (blocks of one query tile, dealt out beforehand)
    __device__ __forceinline__ int next() const { return more[of_blocks<M> ? 1 : 0].w; }
    // slots of the item's sequence, and the row of its first query
    __device__ __forceinline__ int n(const PrefillArgs& a) const { return of_blocks<M> ? more[0].z : a.n; }
    __device__ __forceinline__ int q_row(const Item& it) const { return of_blocks<M> ? more[0].x : it.pos_lo; }
};

// A CTA's own item and the first records of its loads, in the producer's lanes.
template <int D, int M>
struct FirstItem {
    ItemRecord<M> item;
    int4 rec;         // (one sequence's prefill)
    BlockBatch<D, M> batch;  // (block items)
    __device__ void read(const PrefillArgs& a, int w, int lane) {
        item.read(a, blockIdx.x);
        if constexpr (of_blocks<M>) batch.read(a, make_item<M>(a, item.raw), 0, w, lane);
        else rec = tile_record(a, item.raw.y, item.raw.z, 0, lane);
    }
};

// K_0 and K_1 of a CTA's own dual-key item, before the grid-dependency wait:
// unless a page of theirs may still be being written, or one has rows past the
// sequence's end.  Returns the loads issued (2 or 0).  Two of the ring's slots
// and not all: where nothing precedes the launch, the queries, whose load waits
// for the dependency, would queue behind the ring's 20 MB (8 queries over
// 131,080 tokens: calls apart 90.4 us with four loads, 89.3 with two or none;
// layers back to back 85.4, 85.4 and 86.3).
template <int D, int M>
__device__ __forceinline__ int early_loads(const CUtensorMap* pool_map, const PrefillShortArgs& a,
                                           const Smem& sm, const FirstItem<D, M>& start, const Item& it,
                                           int lane) {
    using C = PreCfg<D, M>;
    static_assert(C::kSlots > 2, "ring");
    const int32_t unsafe = lane < a.n_unsafe ? a.unsafe[lane] : -1;
    const int j_tail = it.t0 + it.T == a.n_tiles ? it.T - 1 : it.T;
    // lanes 0 and 1 have the records of key tiles 0 and 1
    const int pg0 = start.rec.y, pg1 = start.rec.z;
    bool safe = it.dual && j_tail > 1;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int p0 = __shfl_sync(0xffffffffu, pg0, x), p1 = __shfl_sync(0xffffffffu, pg1, x);
        safe = safe && (uint32_t)p0 < (uint32_t)a.num_pages && (uint32_t)p1 < (uint32_t)a.num_pages;
        safe = safe && !(unsafe >= 0 && (unsafe == p0 || unsafe == p1));
    }
    safe = __all_sync(0xffffffffu, safe);
    __syncwarp();  // (lane 0 initialised the barriers)
    if (safe && lane < 2) {
        const uint32_t fb = sm.bar<D, M>(C::kBarFull + lane);
        const uint32_t dst = sm.base + C::kOffRing + lane * C::kSlotBytes;
        mbar_arrive_expect_tx(fb, C::kSlotBytes);
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int cb = 0; cb < C::kColBlocks; ++cb)
                tma_load_4d(dst + cb * C::kBlockBytes + b * 64 * 128, pool_map, fb, cb * 64,
                            it.g * a.P + ((b ? start.rec.w : start.rec.x) & (a.P - 1)), b ? pg1 : pg0,
                            a.layer);
    }
    __syncwarp();
    return safe ? 2 : 0;
}

// The same for a block item on pages of 64 tokens or more: its first two loads, the
// first four lanes' boxes, or, of two producer warps' loads, the first one's.
template <int D, int M>
__device__ __forceinline__ int early_loads(const CUtensorMap* pool_map, const BlockShortArgs& a,
                                           const Smem& sm, const FirstItem<D, M>& start, const Item& it,
                                           int lane) {
    using C = PreCfg<D, M>;
    const int32_t unsafe = lane < a.n_unsafe ? a.unsafe[lane] : -1;
    constexpr int kBoxes = producers<M> > 1 ? 2 : 4;
    const int32_t page = start.batch.page, key = start.batch.key;
    // (whole boxes inside the sequence)
    bool safe = lane >= kBoxes || ((uint32_t)page < (uint32_t)a.num_pages && key <= start.item.n(a) - 64);
#pragma unroll
    for (int x = 0; x < kBoxes; ++x) {
        const int32_t p = __shfl_sync(0xffffffffu, page, x);  // (every lane's)
        safe = safe && !(unsafe >= 0 && unsafe == p);
    }
    safe = __all_sync(0xffffffffu, safe);
    __syncwarp();  // (lane 0 initialised the barriers)
    if (safe && lane < kBoxes) {
        const int u = lane >> 1;
        int j, kv;
        load_of<s_buffers<D, M>>(u, it.T, it.dual, j, kv);
        const uint32_t fb = sm.bar<D, M>(C::kBarFull + u);
        if (!(lane & 1)) mbar_arrive_expect_tx(fb, C::kSlotBytes);
        __syncwarp((1u << kBoxes) - 1);
#pragma unroll
        for (int cb = 0; cb < C::kColBlocks; ++cb)
            tma_load_4d(sm.base + C::kOffRing + u * C::kSlotBytes + cb * C::kBlockBytes + (lane & 1) * 64 * 128,
                        pool_map, fb, cb * 64, (kv ? a.Hkv + it.g : it.g) * a.P + (key & (a.P - 1)), page,
                        a.layer);
    }
    __syncwarp();
    return safe ? kBoxes / 2 : 0;
}

// The producer warp, item by item: the query tiles, then the K and V tiles of
// every key tile into the ring in the order of load_of, two loads at a time:
// the whole warp waits for both slots, then lanes 0 and 1 arm their barriers
// and issue their copies together, so that the shared-memory round trips of
// the two overlap.  The queries of an item wait until the previous item's last
// QK product is done; its first two loads go out before that wait.  What a
// tile's copies need, {first key, page of box 0, page of box 1}, is held in
// registers: lane l has the record of the window's key tile j = l (mod 32),
// batches of 16 tiles alternating between the lower and the upper half-warp;
// a batch is read from global memory about ten tiles before its first use and
// moved into place a few tiles before it, an item's first batch while the item
// before it runs.  Boxes past the second (pages of fewer than 64 tokens) take
// their page from global memory.
template <int D, int M>
__device__ void prefill_produce(const CUtensorMap* pool_map, const CUtensorMap* qmap,
                                const PrefillArgs& a, const Smem& sm, const FirstItem<D, M>& start,
                                int u_early, volatile int* abort_flag, int lane) {
    using C = PreCfg<D, M>;
    const int br = a.P < 64 ? a.P : 64;  // rows of one TMA box
    const int n_pieces = a.n_pieces;      // <= 16
    auto load_rec = [&](int t0, int T, int tb) { return tile_record(a, t0, T, tb, lane); };
    int4 raw = start.item.raw, first = start.rec;  // the item, and its first batch of records
    uint32_t n_items = 1;     // items published (the first at start-up)
    bool asked = false;       // an answer of the launch hardware is due
    uint32_t ub = 0;          // loads issued before this item (even)
    uint32_t n_queries = 0;   // items whose queries were loaded
    uint32_t n_fix = 0;       // uses of the fix-up barrier
    uint32_t issued = u_early;
    // Slots are freed by the MMA warp's commits: one for every V tile, which
    // covers the K tile loaded right after it too, and one for each item's
    // first K tile; in dual-key mode one for every tile.  Bit i of `own`: the
    // load i + 1 before the next one has a commit of its own; bit s of `par`:
    // parity of slot s's next commit.
    uint32_t own = 0, par = 0;
    uint32_t slot0 = u_early;  // slot of the next load
    uint32_t tail_u = 0;      // the load that used the fix-up barrier last
    bool tail_open = false;   // ... and was not handed over on its slot's barrier
    bool ok = true;
    auto load_queries = [&](const Item& it) {
        if (n_queries > 0)
            ok = mbar_wait(sm.bar<D, M>(C::kBarQFree), (n_queries - 1) & 1, abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        if (ok && lane == 0) {
            const int nq = it.two ? 2 : 1;  // tile b is loaded only when it holds queries
            mbar_arrive_expect_tx(sm.bar<D, M>(C::kBarQ), nq * C::kColBlocks * a.BP * a.G * 128);
            for (int t = 0; t < nq; ++t)
                for (int cb = 0; cb < C::kColBlocks; ++cb)
                    tma_load_3d(sm.base + C::kOffQ + t * C::kQBytes + cb * C::kBlockBytes, qmap,
                                sm.bar<D, M>(C::kBarQ), cb * 64, it.g * a.G, it.pos_lo + t * a.BP);
        }
        if (ok) ++n_queries;
    };
    // hands an item (or the end mark) to the other roles
    auto publish = [&](int4 r) {
        const int slot = n_items % kItemSlots;
        if (n_items >= kItemSlots)
            ok = __all_sync(0xffffffffu,
                            mbar_wait(sm.bar<D, M>(C::kBarItemFree + slot),
                                      (n_items / kItemSlots - 1) & 1, abort_flag));
        if (ok && lane == 0) {
            *reinterpret_cast<int4*>(sm.ptr + C::kOffItems + slot * 16) = r;
            mbar_arrive(sm.bar<D, M>(C::kBarItem + slot));
        }
        if (ok) ++n_items;
    };
    // The next item: requested six key tiles before an item's end, as late as
    // the answer and its records allow, so that the SMs that are ahead take the
    // items left (asking with the first loads gave them out an item early: 3,001
    // queries over 33,001 tokens 841 -> 835 us); taken in with the last loads.
    int4 next = make_int4(0, 0, -1, 0);
    auto request = [&]() {
        if (lane == 0) {
            mbar_arrive_expect_tx(sm.bar<D, M>(C::kBarClc), 16);
            clc_request(sm.base + C::kOffClc, sm.bar<D, M>(C::kBarClc));
        }
        asked = true;
    };
    auto take_next = [&](uint32_t parity) {
        ok = __all_sync(0xffffffffu, mbar_wait(sm.bar<D, M>(C::kBarClc), parity, abort_flag));
        if (!ok) return;
        asked = false;
        const int cta = clc_answer(sm.base + C::kOffClc);
        next = make_int4(0, 0, -1, 0);
        if (cta >= 0 && cta < a.n_items)
            next = __ldg(reinterpret_cast<const int4*>(a.items) + cta);
        first = load_rec(next.y, next.z, 0);
        // the answer's words are read before the next request overwrites them
        fence_proxy_async_smem();
        __syncwarp();
    };
    if (u_early > 0) own = 3;  // as the loop below keeps it
    while (ok && raw.z >= 0) {
        const Item it = make_item<M>(a, raw);
        const uint32_t clc_parity = (n_items - 1) & 1;
        int4 rec = first, pend = first;
        const int T = it.T;
        const int n_units = 2 * T;
        const int take_at = n_units - 2, ask_at = n_units > 14 ? n_units - 12 : 0;
        const bool late_queries = ub > 0;
        if (T > 0 && !late_queries) load_queries(it);
        if (u_early > ask_at) request();
        if (T == 0) {
            request();
            take_next(clc_parity);
        }
        int fill_b = 1;    // the next batch to read
        int merge_b = -1;  // the batch read into `pend`, not yet in place
        // only the sequence's last key tile has rows past its end
        const int j_tail = it.t0 + T == a.n_tiles ? T - 1 : T;
        for (int u0 = u_early; ok && u0 < n_units; u0 += 2) {  // n_units is even
            int j0, kv0, j1, kv1;
            load_of(u0, T, it.dual, j0, kv0);
            load_of(u0 + 1, T, it.dual, j1, kv1);
            const int jmax = j0 > j1 ? j0 : j1;
            if (merge_b >= 0 && jmax + 4 >= kBatch * merge_b) {
                if ((lane >> 4) == (merge_b & 1)) rec = pend;
                merge_b = -1;
            }
            if (merge_b < 0 && fill_b * kBatch < T && jmax + 10 >= kBatch * fill_b) {
                if ((lane >> 4) == (fill_b & 1)) pend = load_rec(it.t0, T, fill_b * kBatch);
                merge_b = fill_b++;
            }
            const uint32_t U0 = ub + u0;
            const uint32_t slot1 = slot0 + 1 == C::kSlots ? 0 : slot0 + 1;
            const int j = (lane & 1) ? j1 : j0, kv = (lane & 1) ? kv1 : kv0;
            const int key0 = __shfl_sync(0xffffffffu, rec.x, j & 31);
            const int pg0 = __shfl_sync(0xffffffffu, rec.y, j & 31);
            const int pg1 = __shfl_sync(0xffffffffu, rec.z, j & 31);
            const int key0b = __shfl_sync(0xffffffffu, rec.w, j & 31);
            const int slot = (lane & 1) ? slot1 : slot0;  // lanes 0 and 1 issue
            const uint32_t dst = sm.base + C::kOffRing + slot * C::kSlotBytes;
            const int head_row = (kv ? a.Hkv + it.g : it.g) * a.P;
            // every lane polls the slots' barriers in turn: warp-uniform waits,
            // so no lane waits at the vote below for two polling lanes
            if (U0 >= C::kSlots && ((own >> (C::kSlots - 1)) & 1u)) {
                ok = mbar_wait(sm.bar<D, M>(C::kBarEmpty + slot0), (par >> slot0) & 1u, abort_flag);
                par ^= 1u << slot0;
            }
            if (U0 + 1 >= C::kSlots && ((own >> (C::kSlots - 2)) & 1u)) {
                if (ok)
                    ok = mbar_wait(sm.bar<D, M>(C::kBarEmpty + slot1), (par >> slot1) & 1u, abort_flag);
                par ^= 1u << slot1;
            }
            own = own << 2 | (it.dual || j0 == 0 ? 3u : 1u);  // K_j0, V_j1 but in dual-key mode
            // both slots free, or neither load is issued
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            auto checked = [&](int32_t page) {
                if ((uint32_t)page < (uint32_t)a.num_pages) return page;
                // a page outside the pool: flagged; the box is read from page 0
                // so that the barrier's byte count still completes
                set_error(a.err, kErrBounds);
                return 0;
            };
            auto load_box = [&](uint32_t bar, int i, int key, int32_t page) {
                const int row = head_row + (key & (a.P - 1));  // P is a power of two
#pragma unroll
                for (int cb = 0; cb < C::kColBlocks; ++cb)
                    tma_load_4d(dst + cb * C::kBlockBytes + i * br * 128, pool_map, bar, cb * 64, row,
                                page, a.layer);
            };
            if (n_pieces == 2 && jmax < j_tail) {
                // two whole boxes of 64 rows, as almost every tile has
                if (lane < 2) {
                    const uint32_t fb = sm.bar<D, M>(C::kBarFull + slot);
                    mbar_arrive_expect_tx(fb, C::kSlotBytes);
                    load_box(fb, 0, key0, checked(pg0));
                    load_box(fb, 1, key0b, checked(pg1));
                }
            } else {
                // rows of the tile inside the sequence: the lower half's, then
                // the upper half's
                const int rows_b = key0b < a.n ? min(64, a.n - key0b) : 0;
                const int rows = rows_b > 0 ? 64 + rows_b : min(64, a.n - key0);
                const bool vfix = lane < 2 && kv == 1 && rows < kPrefillKeys;
                if (lane < 2) {
                    const int nv = (rows + br - 1) / br;  // boxes inside the sequence (a prefix)
                    const uint32_t fb = vfix ? sm.bar<D, M>(C::kBarVfix) : sm.bar<D, M>(C::kBarFull + slot);
                    mbar_arrive_expect_tx(fb, (uint32_t)nv * br * 128 * C::kColBlocks);
                    const int half = n_pieces / 2;
#pragma unroll 1
                    for (int i = 0; i < nv; ++i) {
                        const int32_t page =
                            i == 0
                                ? pg0
                                : (i == 1 ? pg1
                                          : __ldg(&a.tile_pages[(size_t)(it.t0 + j) * n_pieces + i]));
                        load_box(fb, i, i < half ? key0 + i * br : key0b + (i - half) * br,
                                 checked(page));
                    }
                }
                const uint32_t fix = __ballot_sync(0xffffffffu, vfix);
                if (fix) {
                    // V of the last key tile: its rows past the sequence's end hold
                    // stale or never-written data.  Their weights are zero, but
                    // 0 * NaN is not, so zero those rows before the MMAs read the slot.
                    const int src = __ffs(fix) - 1;
                    const int fslot = __shfl_sync(0xffffffffu, slot, src);
                    const int r0 = __shfl_sync(0xffffffffu, rows, src);  // 1 .. 127
                    tail_u = U0 + src;
                    tail_open = true;
                    issued = U0 + 2;
                    if (lane == 0) ok = mbar_wait(sm.bar<D, M>(C::kBarVfix), n_fix & 1, abort_flag);
                    ok = __shfl_sync(0xffffffffu, ok ? 1 : 0, 0);
                    if (!ok) break;
                    ++n_fix;
                    const int chunks = (kPrefillKeys - r0) * 8;
                    uint8_t* vsp = sm.ptr + C::kOffRing + fslot * C::kSlotBytes;
                    for (int cb = 0; cb < C::kColBlocks; ++cb)
                        for (int c = lane; c < chunks; c += 32)
                            *reinterpret_cast<uint4*>(vsp + cb * C::kBlockBytes +
                                                      (r0 + (c >> 3)) * 128 + (c & 7) * 16) =
                                make_uint4(0, 0, 0, 0);
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(sm.bar<D, M>(C::kBarFull + fslot));
                    tail_open = false;
                }
            }
            issued = U0 + 2;
            slot0 = slot1 + 1 == C::kSlots ? 0 : slot1 + 1;
            if (u0 == ask_at) request();
            if (u0 == 0 && late_queries) load_queries(it);
            if (ok && u0 == take_at) take_next(clc_parity);
        }
        ub += n_units;
        u_early = 0;
        raw = next;
        if (ok) publish(raw);  // an item, or the end mark
    }
    if (!ok && lane == 0) {
        if (!*abort_flag) set_error(a.err, kErrTimeout);
        *abort_flag = 1;
    }
    // Drain: every copy this CTA issued lands before the CTA exits (immediate
    // unless a consumer gave up early).
    if (lane == 0) {
        if (asked) mbar_wait(sm.bar<D, M>(C::kBarClc), (n_items - 1) & 1);
        if (n_queries > 0) mbar_wait(sm.bar<D, M>(C::kBarQ), (n_queries - 1) & 1);
        for (uint32_t u = issued > C::kSlots ? issued - C::kSlots : 0; u < issued; ++u) {
            if (u == tail_u && tail_open) mbar_wait(sm.bar<D, M>(C::kBarVfix), n_fix & 1);
            else mbar_wait(sm.bar<D, M>(C::kBarFull + u % C::kSlots), (u / C::kSlots) & 1);
        }
    }
}

// Load b of a batch (see block_produce, whose lanes hold a box each) for rows in 8 bits:
// its boxes of codes, with their scales, and for the converters the rows of V that the
// sequence has.  Pages of 64 tokens or more: two boxes with 32 bytes of scales each,
// issued by one elected thread.  (Every lane with a box issuing its own, and a scale
// by cp.async for each lane, took 1,400 cycles a load.)  Else a lane to each box and to
// the scale of each eight rows: a box has less of them than a bulk copy takes.
template <int D, int M, typename Args>
__device__ __forceinline__ void issue_codes(const CUtensorMap* pool_map, const Args& a, const Smem& sm, uint32_t bar,
                                            uint32_t slot, int b, int per, int mine, int piece, int32_t page, int row,
                                            int rows, uint32_t bytes, int kv, int lane) {
    using C = PreCfg<D, M>;
    const uint32_t codes = sm.base + C::kOffCodes + slot * C::kCodeStride;
    const uint32_t scales = sm.base + C::kOffScales + slot * C::kTileScales * 4;
    volatile int* n_rows = reinterpret_cast<volatile int*>(sm.ptr + C::kOffRows + 4 * slot);
    const int64_t page_rows = (int64_t)2 * a.Hkv * a.P, layer_row = (int64_t)a.layer * a.num_pages * page_rows;
    constexpr uint32_t kBoxScales = 64 / kScaleRows * 4;  // bytes
    if (per == 2) {
        const int from = 2 * b;
        const int32_t p0 = __shfl_sync(0xffffffffu, page, from), p1 = __shfl_sync(0xffffffffu, page, from + 1);
        const int w0 = __shfl_sync(0xffffffffu, row, from), w1 = __shfl_sync(0xffffffffu, row, from + 1);
        const int limit = kv == 1 ? rows : 64;
        const int r = __shfl_sync(0xffffffffu, limit, from) + __shfl_sync(0xffffffffu, limit, from + 1);
        if (elect_one()) {
            *n_rows = r;
            const uint32_t n = (p0 >= 0 ? 1 : 0) + (p1 >= 0 ? 1 : 0);
            mbar_arrive_expect_tx(bar, n * (64 * D + kBoxScales));
            if (p0 >= 0) {
                tma_load_4d(codes, pool_map, bar, 0, w0, p0, a.layer);
                bulk_load(scales, a.scales + (layer_row + p0 * page_rows + w0) / kScaleRows, kBoxScales, bar);
            }
            if (p1 >= 0) {
                tma_load_4d(codes + 64 * D, pool_map, bar, 0, w1, p1, a.layer);
                bulk_load(scales + kBoxScales, a.scales + (layer_row + p1 * page_rows + w1) / kScaleRows, kBoxScales,
                          bar);
            }
        }
        __syncwarp();
        return;
    }
    const int br = 128 / per;
    const int r = __reduce_add_sync(0xffffffffu, mine == b ? rows : 0);
    // the lane's eight rows lie in lane `from`'s box
    const int from = b * per + lane * kScaleRows / br;
    const int32_t spage = __shfl_sync(0xffffffffu, page, from & 31);
    const int srow = __shfl_sync(0xffffffffu, row, from & 31) + lane * kScaleRows % br;
    if (mine == b) {
        if (piece == 0) {
            *n_rows = kv == 1 ? r : kPrefillKeys;
            mbar_arrive_expect_tx(bar, bytes);
        }
        __syncwarp((uint32_t)((1ull << per) - 1) << (b * per));
        if (page >= 0) tma_load_4d(codes + piece * br * D, pool_map, bar, 0, row, page, a.layer);
    }
    __syncwarp();
    if (lane < C::kTileScales) {
        if (spage >= 0)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(scales + lane * 4),
                         "l"(a.scales + (layer_row + spage * page_rows + srow) / kScaleRows)
                         : "memory");
        // (arrives when this lane's copy has landed)
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
    }
}

// The producer warps of block items.  A lane holds what one box of the next loads
// needs (BlockBatch), so that a load costs a warp a wait, an expected byte count and
// the boxes' copies.  Pages of 64 tokens or more are one warp's loads (one-tile blocks
// of 64 dimensions: two warps', 108 -> 99 us for 8 trees of 16 over 32,768 tokens at
// 64/8/64 heads, where one warp is the bound).  Smaller pages
// have 4, 8 or 16 boxes a load; there the even loads are one warp's, the odd ones
// the other's, and every load's slot has a commit of its own (8 trees of 16 over
// 32,768 tokens on pages of 16 and 8 tokens, 4 and 8 KV heads of 64 dimensions: 83 ->
// 60 and 221 -> 136 us; with two warps on pages of 64 tokens the issuing lane, which
// bounds two-tile items, ran 3% slower).  The first warp (w = 0) also loads the
// queries and takes the next item a few loads before the end of this one; either
// reads its next records then.
template <int D, int M, typename Args>
__device__ void block_produce(const CUtensorMap* pool_map, const CUtensorMap* qmap, const Args& a,
                              const Smem& sm, const FirstItem<D, M>& start, int early,
                              volatile int* abort_flag, int w, int lane) {
    using C = PreCfg<D, M>;
    // blocks of one tile are dealt out to the CTAs beforehand: HBM bounds them, and
    // an even share of the bytes beats handing out whole items
    constexpr bool kDealt = one_tile<M>;
    constexpr int kWarps = producers<M>;
    const int per = pieces_of<M>(a), br = 128 / per;
    const int n_batch = 32 / per;  // loads of a batch
    const int mine = lane / per, piece = lane & (per - 1);
    const uint32_t group = (uint32_t)((1ull << per) - 1);
    ItemRecord<M> item = start.item, next = start.item;
    BlockBatch<D, M> first = start.batch;
    uint32_t k = 0;           // the item's number
    bool asked = false;       // an answer of the launch hardware is due
    uint32_t n_queries = 0;   // items whose queries were loaded
    uint32_t issued = 0;      // this warp's loads
    uint32_t slot = w, phase = 0;  // of its next load
    // (one warp: slots are freed as in prefill_produce)
    uint32_t own = early > 0 ? 3 : 0, par = 0;
    uint32_t n_fix = 0;       // uses of the fix-up barrier
    bool tail_open = false;   // the last load's V is still to be handed over
    bool ok = true;
    auto load_queries = [&](const Item& it) {
        if (k > 0) ok = mbar_wait(sm.bar<D, M>(C::kBarQFree), (k - 1) & 1, abort_flag);
        ok = __all_sync(0xffffffffu, ok);
        if (ok && lane == 0) {
            const int nq = it.two ? 2 : 1;  // tile b is loaded only when it holds queries
            mbar_arrive_expect_tx(sm.bar<D, M>(C::kBarQ), nq * C::kColBlocks * a.BP * a.G * 128);
            for (int t = 0; t < nq; ++t)
                for (int cb = 0; cb < C::kColBlocks; ++cb)
                    tma_load_3d(sm.base + C::kOffQ + t * C::kQBytes + cb * C::kBlockBytes, qmap,
                                sm.bar<D, M>(C::kBarQ), cb * 64, it.g * a.G, item.q_row(it) + t * a.BP);
        }
        if (ok) ++n_queries;
    };
    // The first warp asks for the item after this one, and hands it (or the end
    // mark) to the other roles; the second waits for it.
    auto request = [&]() {
        if constexpr (!kDealt) {
            if (lane == 0) {
                mbar_arrive_expect_tx(sm.bar<D, M>(C::kBarClc), 16);
                clc_request(sm.base + C::kOffClc, sm.bar<D, M>(C::kBarClc));
            }
            asked = true;
        }
    };
    auto take_next = [&]() {
        const uint32_t at = (k + 1) % kItemSlots;
        if (w == 1) {
            ok = __all_sync(0xffffffffu, item_wait<D, M>(sm, k + 1, abort_flag));
            if (!ok) return;
            next.copy(sm.ptr + C::kOffItems + at * C::kItemBytes);
            __syncwarp();
            if (lane == 0) item_free<D, M>(sm, k + 1);
            return;
        }
        int index;
        if constexpr (kDealt) {
            index = item.next();
        } else {
            ok = __all_sync(0xffffffffu, mbar_wait(sm.bar<D, M>(C::kBarClc), k & 1, abort_flag));
            if (!ok) return;
            asked = false;
            const int cta = clc_answer(sm.base + C::kOffClc);
            index = cta < a.n_items ? cta : -1;
            // the answer's words are read before the next request overwrites them
            fence_proxy_async_smem();
            __syncwarp();
        }
        next.raw = make_int4(0, 0, -1, 0);
        if (index >= 0) next.read(a, index);
        if (k + 1 >= kItemSlots)
            ok = __all_sync(0xffffffffu, mbar_wait(sm.bar<D, M>(C::kBarItemFree + at),
                                                   ((k + 1) / kItemSlots - 1) & 1, abort_flag));
        if (ok && lane == 0) {
            next.write(sm.ptr + C::kOffItems + at * C::kItemBytes);
            mbar_arrive(sm.bar<D, M>(C::kBarItem + at));
        }
    };
    if (kWarps > 1 && w == 1 && lane == 0) item_free<D, M>(sm, 0);  // (its first item it has read itself)
    for (; ok && item.raw.z >= 0; ++k) {
        const Item it = make_item<M>(a, item.raw);
        const int n = item.n(a), T = 2 * it.T / kWarps;  // this warp's loads of the item
        // (the second warp waits for the item only after loads that the first one's
        // way there may depend on)
        const int ask_at = max(T - 14 / kWarps, 0), take_at = max(w ? T - 2 : T - 8 / kWarps, 0),
                  read_at = max(T - 4 / kWarps, 0), query_at = kWarps == 2 ? 0 : 1;
        if (w == 0 && k == 0) load_queries(it);
        BlockBatch<D, M> cur = first, ahead;
        for (int x0 = 0; ok && x0 < T; x0 += n_batch) {
            ahead.read(a, it, x0 + n_batch, w, lane);
            // this lane's box
            int j, kv;
            load_of<s_buffers<D, M>>(min(x0 + mine, T - 1) * kWarps + w, it.T, it.dual, j, kv);
            const bool box = cur.page >= 0;
            const uint32_t boxes = __ballot_sync(0xffffffffu, box) >> (mine * per) & group;
            const uint32_t bytes = (uint32_t)__popc(boxes) * br * (e8<M> ? D : 128 * C::kColBlocks);
            const int rows = box ? min(br, n - cur.key) : 0;  // rows of the sequence in the box
            // V of the sequence's last key tile (an odd load): its rows past the end
            // are zeroed
            const uint32_t fixes = __ballot_sync(0xffffffffu, kv == 1 && rows < br && x0 + mine < T);
            const int row = (kv ? a.Hkv + it.g : it.g) * a.P + (cur.key & (a.P - 1));  // P is a power of two
            int32_t page = cur.page;
            if (box && page >= a.num_pages) {
                // a page outside the pool: flagged; the box is read from page 0 so
                // that the barrier's byte count still completes
                set_error(a.err, kErrBounds);
                page = 0;
            }
            const int last = min(n_batch, T - x0);
            for (int b = 0; b < last; ++b) {
                const int x = x0 + b;
                if ((int)issued < early) {
                    // (the first loads went out before the dependency wait)
                } else {
                    const uint32_t empty = sm.bar<D, M>(C::kBarEmpty + slot);
                    // every lane polls the slot's barrier: a warp-uniform wait
                    if (kWarps * issued + w >= C::kSlots && (kWarps > 1 || ((own >> (C::kSlots - 1)) & 1u))) {
                        const uint32_t parity = kWarps > 1 ? phase ^ 1 : (par >> slot) & 1u;
                        ok = __all_sync(0xffffffffu, mbar_wait(empty, parity, abort_flag));
                        par ^= 1u << slot;
                        if (!ok) break;
                    }
                    own = own << 1 | (it.dual || (x & 1) || x == 0 ? 1u : 0u);
                    const uint32_t fix = e8<M> ? 0u : fixes >> (b * per) & group;
                    const uint32_t bar = e8<M> ? sm.bar<D, M>(C::kBarRaw + slot)
                                         : fix ? sm.bar<D, M>(C::kBarVfix)
                                               : sm.bar<D, M>(C::kBarFull + slot);
                    if constexpr (e8<M>)
                        issue_codes<D, M>(pool_map, a, sm, bar, slot, b, per, mine, piece, page, row, rows, bytes, kv,
                                          lane);
                    if (!e8<M> && mine == b) {
                        if (piece == 0) mbar_arrive_expect_tx(bar, bytes);
                        __syncwarp(group << (b * per));
                        if (box) {
                            const uint32_t dst =
                                sm.base + C::kOffRing + slot * C::kSlotBytes + piece * br * 128;
#pragma unroll
                            for (int cb = 0; cb < C::kColBlocks; ++cb)
                                tma_load_4d(dst + cb * C::kBlockBytes, pool_map, bar, cb * 64, row, page,
                                            a.layer);
                        }
                    }
                    if (fix) {
                        // stale or never-written data: their weights are zero, but
                        // 0 * NaN is not, so the rows are zeroed before the MMAs read
                        // them
                        tail_open = true;
                        ++issued;
                        const int r0 = __reduce_add_sync(0xffffffffu, mine == b ? rows : 0);
                        ok = __all_sync(0xffffffffu,
                                        mbar_wait(sm.bar<D, M>(C::kBarVfix), n_fix & 1, abort_flag));
                        if (!ok) break;
                        --issued;
                        ++n_fix;
                        const int chunks = (kPrefillKeys - r0) * 8;
                        uint8_t* vsp = sm.ptr + C::kOffRing + slot * C::kSlotBytes;
                        for (int cb = 0; cb < C::kColBlocks; ++cb)
                            for (int c = lane; c < chunks; c += 32)
                                *reinterpret_cast<uint4*>(vsp + cb * C::kBlockBytes + (r0 + (c >> 3)) * 128 +
                                                          (c & 7) * 16) = make_uint4(0, 0, 0, 0);
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(sm.bar<D, M>(C::kBarFull + slot));
                        tail_open = false;
                    }
                }
                ++issued;
                slot += kWarps;
                if (slot >= C::kSlots) {
                    slot -= C::kSlots;
                    phase ^= 1;
                }
                if (w == 0) {
                    if (x == ask_at) request();
                    if (x == query_at && k > 0) load_queries(it);
                }
                if (x == take_at) take_next();
                if (x == read_at && ok) first.read(a, make_item<M>(a, next.raw), 0, w, lane);
                if (!ok) break;
            }
            cur = ahead;
        }
        if (ok) item = next;
    }
    if (!ok && lane == 0) {
        if (!*abort_flag) set_error(a.err, kErrTimeout);
        *abort_flag = 1;
    }
    // Drain: every copy this warp issued lands before the CTA exits (immediate
    // unless a consumer gave up early).  Of the last kSlots loads (either warp has
    // issued as many) the slots were not filled again, by the other warp either,
    // so their barriers still are in the phase waited for.
    if (lane == 0) {
        if (asked) mbar_wait(sm.bar<D, M>(C::kBarClc), (k - 1) & 1);
        if (n_queries > 0) mbar_wait(sm.bar<D, M>(C::kBarQ), (n_queries - 1) & 1);
        const uint32_t total = kWarps * issued;
        for (uint32_t x = total > C::kSlots ? (total - C::kSlots + kWarps - 1 - w) / kWarps : 0; x < issued; ++x) {
            const uint32_t U = kWarps * x + w;
            if (tail_open && x + 1 == issued) mbar_wait(sm.bar<D, M>(C::kBarVfix), n_fix & 1);
            else mbar_wait(sm.bar<D, M>((e8<M> ? C::kBarRaw : C::kBarFull) + U % C::kSlots), (U / C::kSlots) & 1);
        }
    }
}

// Registers of each of a warpgroup's threads from here on.
template <int N, bool kMore>
__device__ __forceinline__ void take_registers() {
    if constexpr (kMore) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

// Rows in 8 bits: the converters widen a tile's codes to bf16 where the products read
// them: code times scale, exact, so that everything behind is as for bf16 rows.  A
// thread takes a row, half of it at a time (of 128 codes: what it writes lies over its
// own row's codes alone, which it has read by then).  V rows past the sequence's end are
// zeroed, as the bf16 instances' producer does.  (Eight warps on one tile, half a row a
// thread: 1,600 cycles a tile, most of them the chain of loads, conversions, stores and
// fence, which two groups on a tile each overlap: 107.3 us for 8 trees of 16, 93.0 so.)
//
// A code's conversion makes an fp16 number of it, and one mixed-precision fused
// multiply-add the fp32 product with the scale, where that is an fp16 number.
__device__ __forceinline__ uint32_t widen_pair(uint32_t f16x2, uint16_t scale) {
    float lo, hi;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\t"
        "fma.rn.f32.f16 %0, l, %3, %4;\n\tfma.rn.f32.f16 %1, h, %3, %4;\n\t}"
        : "=f"(lo), "=f"(hi)
        : "r"(f16x2), "h"(scale), "f"(-0.f));
    return pack_bf16x2(lo, hi);
}
// 64 codes of a row as bf16 into its 128 bytes of a column block.
template <bool kNarrow>
__device__ __forceinline__ void widen_half(const uint4 (&c)[4], float s, uint8_t* out, int row) {
    const uint16_t s16 = __half_as_ushort(__float2half_rn(s));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t cw[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t o[4];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t w = cw[2 * h + k];
                if (kNarrow) {
                    o[2 * k] = widen_pair(e4m3_to_f16x2(w), s16);
                    o[2 * k + 1] = widen_pair(e4m3_to_f16x2(w >> 16), s16);
                } else {
                    const float4 v = e4m3_values(w, s);
                    o[2 * k] = pack_bf16x2(v.x, v.y);
                    o[2 * k + 1] = pack_bf16x2(v.z, v.w);
                }
            }
            *reinterpret_cast<uint4*>(out + (((2 * i + h) ^ (row & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
}

template <int D, int M>
__device__ void convert_tiles(const Smem& sm, int* err, volatile int* abort_flag, int w, int lane) {
    using C = PreCfg<D, M>;
    const int row = (w & 3) * 32 + lane, group = w >> 2;
    const int turn = D == 128 ? row & 7 : row >> 1 & 3;  // (the tensor map's swizzle)
    uint32_t slot = group, phase = 0;                    // of the group's next tile
    bool ok = true;
    for (uint32_t k = 0; ok; ++k) {
        ok = __all_sync(0xffffffffu, item_wait<D, M>(sm, k, abort_flag));
        if (!ok) break;
        const int T = item_read<D, M>(sm, k).z;
        __syncwarp();
        if (lane == 0) item_free<D, M>(sm, k);
        if (T < 0) break;
        // (an item's loads are an even number)
        static_assert(kConvertGroups == 2, "a load of either kind of an item's pairs");
        for (int x = 0; x < T; ++x) {
            ok = __all_sync(0xffffffffu, mbar_wait(sm.bar<D, M>(C::kBarRaw + slot), phase, abort_flag));
            if (!ok) break;
            const uint8_t* src = sm.ptr + C::kOffCodes + slot * C::kCodeStride + row * D;
            uint8_t* to = sm.ptr + C::kOffRing + slot * C::kSlotBytes + row * 128;
            const float s =
                reinterpret_cast<const float*>(sm.ptr + C::kOffScales)[slot * C::kTileScales + row / kScaleRows];
            const bool on = row < *reinterpret_cast<const volatile int*>(sm.ptr + C::kOffRows + 4 * slot);
            // (scales are powers of two: most are fp16 numbers too)
            const bool narrow = __all_sync(0xffffffffu, s >= 0x1p-24f && s <= 0x1p15f);
#pragma unroll
            for (int cb = 0; cb < D / 64; ++cb) {
                uint4 c[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    c[i] = *reinterpret_cast<const uint4*>(src + (((cb * 4 + i) ^ turn) << 4));
                uint8_t* out = to + cb * C::kBlockBytes;
                if (narrow) widen_half<true>(c, s, out, row);
                else widen_half<false>(c, s, out, row);
            }
            if (!__all_sync(0xffffffffu, on) && !on)
                for (int x = 0; x < 8 * C::kColBlocks; ++x)
                    *reinterpret_cast<uint4*>(to + (x >> 3) * C::kBlockBytes + (x & 7) * 16) = make_uint4(0, 0, 0, 0);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(sm.bar<D, M>(C::kBarFull + slot));
            slot += kConvertGroups;
            if (slot >= C::kSlots) {
                slot -= C::kSlots;
                phase ^= 1;
            }
        }
    }
    if (!ok && lane == 0) {
        if (!*abort_flag) set_error(err, kErrTimeout);
        *abort_flag = 1;
    }
}

// Descriptors of a CTA's operands: the two query tiles, and the ring's slot 0
// as a K tile (K-major) and as a V tile (MN-major).  Slot s is s *
// kSlotBytes / 16 further in the address field.
struct MmaDesc {
    uint32_t q[2], k, v;      // low words
    uint32_t k_hi, v_hi;      // high words (the queries' is the K tile's)
    uint32_t tmem;
};
template <int D, int M>
__device__ __forceinline__ MmaDesc mma_desc(const Smem& sm, uint32_t tmem) {
    using C = PreCfg<D, M>;
    static_assert(C::kBlockBytes == 16384, "the K-major steps' block stride");
    const uint64_t q = smem_desc_sw128(sm.base + C::kOffQ, 16, 1024);
    const uint64_t k = smem_desc_sw128(sm.base + C::kOffRing, 16, 1024);
    const uint64_t v = smem_desc_sw128(sm.base + C::kOffRing, C::kBlockBytes, 1024);
    MmaDesc d;
    d.q[0] = (uint32_t)q;
    d.q[1] = (uint32_t)q + (C::kQBytes >> 4);
    d.k = (uint32_t)k;
    d.v = (uint32_t)v;
    d.k_hi = (uint32_t)(k >> 32);
    d.v_hi = (uint32_t)(v >> 32);
    d.tmem = tmem;
    return d;
}

// S_t = Q_q K^T for the K tile in `slot`, into S buffer t (q = t except in
// dual-key mode, where both tiles use query tile 0).
template <int D, int M>
__device__ __forceinline__ void issue_qk(const MmaDesc& d, int t, int q, uint32_t slot) {
    using C = PreCfg<D, M>;
    mma_bf16_ss_steps<D / 16>(d.tmem + C::col_s(t), d.q[q],
                              d.k + slot * (C::kSlotBytes >> 4), d.k_hi, C::kIdescQK);
}

// O_t += P_t V for the V tile in `slot`; P_t from TMEM over the first half of S
// buffer `buf` (t where there are two).
template <int D, int M>
__device__ __forceinline__ void issue_pv(const MmaDesc& d, int t, int buf, uint32_t slot, bool first) {
    using C = PreCfg<D, M>;
    static_assert(kPrefillKeys == 128, "8 steps of 16 keys");
    mma_bf16_ts_steps8(d.tmem + C::kColO + (uint32_t)t * C::kOStep, d.tmem + C::col_s(buf),
                       d.v + slot * (C::kSlotBytes >> 4), d.v_hi, C::kIdescPV, first ? 0u : 1u);
}

// Phases of the barriers the MMA warp waits on, running on from item to item.
struct MmaPhase {
    uint32_t ub;    // loads of the items before (K_j, V_j: load_of)
    uint32_t slot;  // ub mod kSlots
    uint32_t p;     // bit t: parity of the next P_t hand-off
    uint32_t q;     // items whose queries were used
};

// The lane that issues the MMAs is the busiest thread of the kernel: whatever
// it does between two products, the tensor core's short queue drains.  So it
// waits for P_t alone: a softmax warp of tile a hands over P only when V_j and
// K_{j+1} have landed too, and one commit after the second PV frees V_j and,
// with it, the K tile used by the QK products issued just before.  (With its
// own waits for both tiles and a commit for each slot the lane needed 3,434
// cycles per key tile for products of 2,650, and was never waiting for P.)
// In dual-key mode memory is the bound, not this lane: it waits for each tile
// by itself and frees each slot at once.
//
// Dual-key mode (every query of the CTA tile fits in tile a): both tiles
// hold tile a's queries; tile a takes key tiles 0, 2, 4, ... and tile b the
// odd ones, and the two results are merged at the end.  Key tile j's PV and
// the QK of key tile j + 2 (into the same S columns) are issued in the order
// of the loads, each as soon as its tile has landed.
template <int D, int M>
__device__ bool prefill_mma_dual(const Smem& sm, const MmaDesc& d, int T, MmaPhase& ph,
                                 volatile int* abort_flag) {
    using C = PreCfg<D, M>;
    // the tiles are used in the order of their loads: K_0, K_1, V_0, K_2, V_1, ...
    uint32_t slot = ph.slot, full = (ph.ub / C::kSlots) & 1;
    auto landed = [&]() { return mbar_wait(sm.bar<D, M>(C::kBarFull + slot), full, abort_flag); };
    auto used = [&]() {
        mma_commit(sm.bar<D, M>(C::kBarEmpty + slot));
        if (++slot == C::kSlots) {
            slot = 0;
            full ^= 1;
        }
    };
    for (int t = 0; t < 2; ++t) {
        // S_t = Q_a K_t
        if (!landed()) return false;
        issue_qk<D, M>(d, t, 0, slot);
        mma_commit(sm.bar<D, M>(C::kBarS + t));
        used();
    }
    if (T == 2) mma_commit(sm.bar<D, M>(C::kBarQFree));  // the item's last QK
    for (int j = 0; j < T; ++j) {
        const int t = j & 1;
        if (!landed()) return false;
        if (!mbar_wait(sm.bar<D, M>(C::kBarP + t), (ph.p >> t) & 1, abort_flag)) return false;
        ph.p ^= 1u << t;
        tc_fence_after();
        issue_pv<D, M>(d, t, t, slot, j < 2);
        used();
        if (j + 2 >= T) {  // the last key tile of tile t
            mma_commit(sm.bar<D, M>(C::kBarO + t));
            continue;
        }
        if (!landed()) return false;
        issue_qk<D, M>(d, t, 0, slot);
        mma_commit(sm.bar<D, M>(C::kBarS + t));
        used();
        if (j + 3 == T) mma_commit(sm.bar<D, M>(C::kBarQFree));  // the item's last QK
    }
    ph.slot = slot;
    return true;
}

// The same with three S buffers: key tile number u of the CTA's life (the item's
// first is u0) in buffer u mod 3, its phase u / 3; PV_j and the QK of key tile
// j + 3, into the buffer that held P_j, are issued together.
template <int D, int M>
__device__ bool prefill_mma_three(const Smem& sm, const MmaDesc& d, int T, MmaPhase& ph,
                                  volatile int* abort_flag) {
    using C = PreCfg<D, M>;
    uint32_t slot = ph.slot, full = (ph.ub / C::kSlots) & 1;
    auto used = [&]() {
        mma_commit(sm.bar<D, M>(C::kBarEmpty + slot));
        if (++slot == C::kSlots) {
            slot = 0;
            full ^= 1;
        }
    };
    const uint32_t u0 = ph.ub / 2;
    for (int j = 0; j < min(3, T); ++j) {  // S = Q_a K_j
        const uint32_t buf = (u0 + j) % 3;
        if (!mbar_wait(sm.bar<D, M>(C::kBarFull + slot), full, abort_flag)) return false;
        issue_qk<D, M>(d, (int)buf, 0, slot);
        mma_commit(sm.bar<D, M>(C::kBarS + buf));
        used();
    }
    if (T <= 3) mma_commit(sm.bar<D, M>(C::kBarQFree));  // the item's last QK
    uint32_t buf = u0 % 3, parity = (u0 / 3) & 1;
    for (int j = 0; j < T; ++j) {
        const int t = j & 1;
        if (!mbar_wait(sm.bar<D, M>(C::kBarP + buf), parity, abort_flag)) return false;
        tc_fence_after();
        issue_pv<D, M>(d, t, (int)buf, slot, j < 2);
        if (j + 3 < T) {
            used();
            issue_qk<D, M>(d, (int)buf, 0, slot);
            mma_commit(sm.bar<D, M>(C::kBarS + buf));
            used();
            if (j + 4 == T) mma_commit(sm.bar<D, M>(C::kBarQFree));
        } else {
            if (j + 3 == T) mma_commit(sm.bar<D, M>(C::kBarPV));
            if (j + 2 >= T) mma_commit(sm.bar<D, M>(C::kBarO + t));  // the last key tile of tile t
            used();
        }
        if (++buf == 3) {
            buf = 0;
            parity ^= 1;
        }
    }
    ph.slot = slot;
    return true;
}

// One step of the two-tile path: O_t += P_t V_j, then S_t for the next key tile,
// for tile a and then tile b.
template <int D, int M, bool kFirst, bool kMore>
__device__ __forceinline__ bool prefill_mma_step(const Smem& sm, const MmaDesc& d, uint32_t vslot,
                                                 uint32_t kslot, uint32_t pa, uint32_t pb,
                                                 const volatile int* abort_flag) {
    using C = PreCfg<D, M>;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        if (!mbar_wait(sm.bar<D, M>(C::kBarP + t), t ? pb : pa, abort_flag)) return false;
        tc_fence_after();
        issue_pv<D, M>(d, t, t, vslot, kFirst);
        if (kMore) issue_qk<D, M>(d, t, t, kslot);
        mma_commit(sm.bar<D, M>(kMore ? C::kBarS + t : C::kBarO + t));
    }
    mma_commit(sm.bar<D, M>(C::kBarEmpty + vslot));  // V_j, and K_{j+1} with it
    // (two producer warps: on its own, for the warp that waits for it)
    if (producers<M> > 1 && kMore) mma_commit(sm.bar<D, M>(C::kBarEmpty + kslot));
    return true;
}

// `two`: tile b holds query rows (false for an item of one key tile whose rows
// all fit in tile a; tile b's products are then skipped).
template <int D, int M>
__device__ bool prefill_mma_item(const Smem& sm, const MmaDesc& d, int T, bool two, MmaPhase& ph,
                                 volatile int* abort_flag) {
    using C = PreCfg<D, M>;
    auto after = [](uint32_t slot) { return slot + 1 == C::kSlots ? 0u : slot + 1; };
    uint32_t slot = ph.slot;
    if (!mbar_wait(sm.bar<D, M>(C::kBarFull + slot), (ph.ub / C::kSlots) & 1, abort_flag)) return false;
    issue_qk<D, M>(d, 0, 0, slot);
    mma_commit(sm.bar<D, M>(C::kBarS + 0));
    if (two) {
        issue_qk<D, M>(d, 1, 1, slot);
        mma_commit(sm.bar<D, M>(C::kBarS + 1));
    }
    mma_commit(sm.bar<D, M>(C::kBarEmpty + slot));
    uint32_t vslot = after(slot), kslot = after(vslot);
    if (one_tile<M> || !two) {
        mma_commit(sm.bar<D, M>(C::kBarQFree));
        if (!mbar_wait(sm.bar<D, M>(C::kBarP + 0), ph.p & 1, abort_flag)) return false;
        tc_fence_after();
        issue_pv<D, M>(d, 0, 0, vslot, true);
        mma_commit(sm.bar<D, M>(C::kBarO + 0));
        mma_commit(sm.bar<D, M>(C::kBarEmpty + vslot));
        ph.p ^= 1u;
        ph.slot = kslot;
        return true;
    }
    uint32_t pa = ph.p & 1, pb = (ph.p >> 1) & 1;
    if (T == 1) {
        mma_commit(sm.bar<D, M>(C::kBarQFree));
        if (!prefill_mma_step<D, M, true, false>(sm, d, vslot, kslot, pa, pb, abort_flag)) return false;
    } else {
        if (!prefill_mma_step<D, M, true, true>(sm, d, vslot, kslot, pa, pb, abort_flag)) return false;
        for (int j = 1; j + 1 < T; ++j) {
            vslot = after(kslot);
            kslot = after(vslot);
            pa ^= 1;
            pb ^= 1;
            if (!prefill_mma_step<D, M, false, true>(sm, d, vslot, kslot, pa, pb, abort_flag))
                return false;
        }
        mma_commit(sm.bar<D, M>(C::kBarQFree));  // the item's last QK
        vslot = after(kslot);
        kslot = after(vslot);
        if (!prefill_mma_step<D, M, false, false>(sm, d, vslot, kslot, pa ^ 1, pb ^ 1, abort_flag))
            return false;
    }
    ph.p ^= (T & 1) ? 3u : 0u;
    ph.slot = kslot;
    return true;
}

// The MMA-issuing lane, item by item.  The next item's first S may be issued
// while the softmax warps still write out this one's O: S has columns of its
// own, and the first PV, which overwrites O, waits for a P that each softmax
// thread hands over only after it has read its O.
template <int D, int M>
__device__ void prefill_mma(const PrefillArgs& a, const Smem& sm, uint32_t tmem,
                            volatile int* abort_flag) {
    using C = PreCfg<D, M>;
    MmaPhase ph = {0, 0, 0, 0};
    const MmaDesc d = mma_desc<D, M>(sm, tmem);
    bool ok = true, any = false;
    for (uint32_t k = 0;; ++k) {
        if (!(ok = item_wait<D, M>(sm, k, abort_flag))) break;
        const int4 raw = item_read<D, M>(sm, k);
        item_free<D, M>(sm, k);
        if (raw.z < 0) break;
        if (raw.z == 0) continue;
        const Item it = make_item<M>(a, raw);
        if (!(ok = mbar_wait(sm.bar<D, M>(C::kBarQ), ph.q & 1, abort_flag))) break;
        tc_fence_after();
        ++ph.q;
        any = true;
        if constexpr (C::kBufs > 2)  // (an item of one key tile as well)
            ok = prefill_mma_three<D, M>(sm, d, it.T, ph, abort_flag);
        else
            ok = it.dual ? prefill_mma_dual<D, M>(sm, d, it.T, ph, abort_flag)
                         : prefill_mma_item<D, M>(sm, d, it.T, it.two, ph, abort_flag);
        if (!ok) break;
        ph.ub += 2 * it.T;
    }
    if (!ok) {
        set_error(a.err, kErrTimeout);
        *abort_flag = 1;
    }
    if (any) {
        // every MMA issued here completes before TMEM is released
        mma_commit(sm.bar<D, M>(C::kBarDone));
        mbar_wait(sm.bar<D, M>(C::kBarDone), 0);
    }
}

// Packed fp32 pair helpers (sm_100 family): d = a * b + c on two lanes at once.
__device__ __forceinline__ uint64_t f2pack(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void f2unpack(uint64_t v, float& lo, float& hi) {
    asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t ffma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
// lo += the low bf16 of w, hi += its high bf16 (mixed-precision adds: the
// bf16 operands are exact in fp32).
__device__ __forceinline__ void add_bf16x2_f32(uint32_t w, float& lo, float& hi) {
    asm("{\n\t.reg .b16 l16, h16;\n\tmov.b32 {l16, h16}, %2;\n\t"
        "add.rn.f32.bf16 %0, l16, %0;\n\tadd.rn.f32.bf16 %1, h16, %1;\n\t}"
        : "+f"(lo), "+f"(hi)
        : "r"(w));
}
// 2^x as the single PTX instruction ex2.approx.ftz (relative error about
// 2^-22).  Results below 2^-126 flush to zero: every row holds a weight of at
// least 1 (its running maximum's), so they change its sums by under 2^-119.
__device__ __forceinline__ float ex2_ftz(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float fmax3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// Every lane of the warp polls the barrier (one instruction for the warp,
// no hand-on from a polling lane: a softmax warp sees its S ready sooner);
// returns the warp-uniform result.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, const volatile int* abort) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort));
}

// Pairs of lanes trade halves of their rows so that each writes 32 bytes of one
// row next to its neighbour's 32: in `own` this lane's 16 words of its row, in
// `out[0]` and `out[1]` afterwards the even and the odd lane's row, the lane's own
// half of the 64 bytes.
__device__ __forceinline__ void trade_halves(const uint32_t (&own)[16], uint32_t (&out)[2][8], bool odd) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t got = __shfl_xor_sync(0xffffffffu, odd ? own[i] : own[8 + i], 1);
        out[0][i] = odd ? got : own[i];
        out[1][i] = odd ? own[8 + i] : got;
    }
}
__device__ __forceinline__ void st_32(void* p, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]),
                 "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}

// Normalises and writes one row of O_t (with tile b's part in dual-key mode) to
// the outputs, or to the item's partial result.  True (blocks): some value of the
// row is an infinity or NaN.
template <int D, int M>
__device__ __forceinline__ bool prefill_write(const PrefillArgs& a, const Item& it, int q_row, uint32_t tl,
                                              uint32_t col_o, int t, int row, bool valid,
                                              float m_run, float l, float wa, float wb) {
    using C = PreCfg<D, M>;
    const bool dual = it.dual, any_keys = it.T > 0;
    const int qi = q_row + (dual ? 0 : t) * a.BP + row / a.G;
    const float inv = l > 0.f ? 1.f / l : 0.f;
    // (a row whose weights are NaN says so, to its merge too)
    const float lse2 = l > 0.f ? m_run + __log2f(l) : (l != 0.f ? NAN : -INFINITY);
    const int h = it.g * a.G + row % a.G;
    float* part_row = nullptr;
    uint8_t* out_row = nullptr;
    if (it.part >= 0) {
        const size_t pr = ((size_t)it.part * kPrefillQTiles + t) * kPrefillRows + row;
        part_row = a.part_o + pr * D;
        if (valid) a.part_ml[pr] = lse2;
    } else {
        out_row = reinterpret_cast<uint8_t*>(a.out) +
                  ((size_t)qi * a.Hq + h) * D * (a.out_f32 ? 4 : 2);
        if (valid && a.lse) a.lse[(size_t)qi * a.Hq + h] = lse2 * 0.69314718055994531f;
    }
    // A block of queries has few key tiles to hide its output behind.  A row for
    // each lane, 16 bytes at a time, takes the store unit a cycle for every row and
    // instruction; where the output allows 32-byte stores, pairs of lanes write 64
    // bytes of one row together (16,384 queries at a window of 1,024: 254 -> 238 us,
    // with the loop rolled up).
    uint8_t* to = part_row ? reinterpret_cast<uint8_t*>(part_row) : out_row;
    const bool paired = of_blocks<M> && (reinterpret_cast<uintptr_t>(a.out) & 31) == 0;
    uint8_t* to_even = nullptr;   // the pair's rows, null: no query
    uint8_t* to_odd = nullptr;
    if (paired) {
        const uint64_t mine = valid ? reinterpret_cast<uint64_t>(to) : 0u;
        const uint64_t other = __shfl_xor_sync(0xffffffffu, mine, 1);
        to_even = reinterpret_cast<uint8_t*>(row & 1 ? other : mine);
        to_odd = reinterpret_cast<uint8_t*>(row & 1 ? mine : other);
    }
    uint64_t odd_values = 0;  // two sums of 0 * value: NaN where one is not finite
    // (a block's: rolled up, for the instruction cache)
#pragma unroll (of_blocks<M> ? 1 : D / 32)
    for (int c = 0; c < D / 32; ++c) {
        uint32_t o[32];
        if (any_keys) {
            tmem_ld32(tl + col_o + c * 32, o);
            tmem_wait_ld();
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = 0u;
        }
        float f[32];
        if (dual) {
            uint32_t ob[32];
            tmem_ld32(tl + C::kColO + C::kOStep + c * 32, ob);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i)
                f[i] = (__uint_as_float(o[i]) * wa + __uint_as_float(ob[i]) * wb) * inv;
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(o[i]) * inv;
        }
        if constexpr (of_blocks<M>) {
#pragma unroll
            for (int i = 0; i < 16; ++i) odd_values = ffma2(f2pack(f[2 * i], f[2 * i + 1]), 0, odd_values);
        }
        if (paired) {
            const bool odd = row & 1;
            uint32_t w[16], x[2][8];
            if (part_row || a.out_f32) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(f[16 * half + i]);
                    trade_halves(w, x, odd);
                    const int at = c * 128 + half * 64 + (odd ? 32 : 0);
                    if (to_even) st_32(to_even + at, x[0]);
                    if (to_odd) st_32(to_odd + at, x[1]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
                trade_halves(w, x, odd);
                const int at = c * 64 + (odd ? 32 : 0);
                if (to_even) st_32(to_even + at, x[0]);
                if (to_odd) st_32(to_odd + at, x[1]);
            }
            continue;
        }
        if (!valid) continue;
        if (part_row || a.out_f32) {
            float4* dst = reinterpret_cast<float4*>(part_row ? part_row + c * 32
                                                             : reinterpret_cast<float*>(out_row) + c * 32);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                dst[i] = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
        } else {
            uint4* dst = reinterpret_cast<uint4*>(out_row + c * 64);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const __nv_bfloat162 hb = __floats2bfloat162_rn(f[8 * i + 2 * e], f[8 * i + 2 * e + 1]);
                    w[e] = *reinterpret_cast<const uint32_t*>(&hb);
                }
                dst[i] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
    float x, y;
    f2unpack(odd_values, x, y);
    return valid && !(x + y == 0.f);
}

// Which keys a row sees, beside the tiles' own visibility bits (positions are
// slots).  In one sequence's prefill: those up to its own.
template <int M>
struct RowMask {
    int p;
    __device__ __forceinline__ void init(const PrefillArgs& a, int qi) { p = a.n - a.n_q + qi; }
    // every one of the 64 keys from k on
    __device__ __forceinline__ bool whole(int k) const { return p - k >= 63; }
    // the 32 keys from k on, a bit each
    __device__ __forceinline__ uint32_t word(int k) const { return low_bits_through(p - k); }
};
// A block item's row sees the keys low .. top and those below the sinks' end, and
// of those from `base` on (a multiple of 32; the drafted tree) what its bitmap
// says.
struct BlockRowMask {
    int low, top, sink_end, base, n_words;
    const uint32_t* bits;
    __device__ __forceinline__ void init(const BlockArgs& a, const BlockItem& it, int qi) {
        if (a.rows) {
            const int2 r = __ldg(a.rows + it.q_row + qi);
            low = r.x;
            top = r.y;
        } else {
            low = it.low0 + qi;
            top = it.pos0 + qi;
        }
        sink_end = it.sink_end;
        base = it.base;
        n_words = a.n_words;
        bits = a.bits + (size_t)(it.q_row + qi) * a.n_words;
    }
    __device__ __forceinline__ bool whole(int k) const {
        return k <= top - 63 && (k >= low || k <= sink_end - 64);
    }
    __device__ __forceinline__ uint32_t word(int k) const {
        if (k >= base) return (k - base) >> 5 < n_words ? __ldg(bits + ((k - base) >> 5)) : 0u;
        return low_bits_through(top - k) &
               (~low_bits_through(low - 1 - k) | low_bits_through(sink_end - 1 - k));
    }
};
template <>
struct RowMask<kBlocks> : BlockRowMask {};
template <>
struct RowMask<kBlocks | kOneTile> : BlockRowMask {};
template <>
struct RowMask<kBlocks | kTwoProducers> : BlockRowMask {};
template <>
struct RowMask<kBlocks | kOneTile | kTwoProducers> : BlockRowMask {};
template <>
struct RowMask<kE8 | kBlocks | kOneTile> : BlockRowMask {};
template <>
struct RowMask<kE8 | kBlocks | kOneTile | kTwoProducers> : BlockRowMask {};

// A key that a row does not see has the weight 0 in the row's tile product, and
// 0 times an infinity or NaN in that key's V row is NaN.  Besides, a row's weights may
// sum to 2^80 (its maximum starts at 0), and times large values they pass
// what fp32 holds where their average is finite.  So where a block's row has an output
// that is not finite though its normaliser is, and some key that its tiles hide has
// such a V row, or no key of the item has one (then the sums overflowed), it is taken
// once more, over the keys that it does see and with the maximum and normaliser that
// it has, the weights divided by the normaliser first, so that every sum is an average
// of values: a warp on four rows of a query at a time, a lane to a key for the weights
// and to D / 32 columns for the sums.  (Sums that overflow beside a key that the row
// sees whose value is not finite stay as they are.)  (An item
// pays D fused multiply-adds a row to look, and nothing more as long as stored rows
// are finite.  A row taken again costs 40 us for 1,000 keys, 130 where a KV head has
// one query head: a warp's 32 rows over 400,000 keys still end within the other
// roles' bounded waits of 2 s.)
//
// Elements 8 c .. 8 c + 7 of a row of the pool (its number in the layer's), and one.
template <int D, int M, typename Args>
__device__ __forceinline__ uint4 pool_eight(const Args& a, int64_t row, int c) {
    row += (int64_t)a.layer * a.num_pages * 2 * a.Hkv * a.P;
    if constexpr (e8<M>) {
        const uint2 x = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.pool) + row * D + 8 * c);
        const float s = __ldg(a.scales + row / kScaleRows);
        const float4 lo = e4m3_values(x.x, s), hi = e4m3_values(x.y, s);
        return make_uint4(pack_bf16x2(lo.x, lo.y), pack_bf16x2(lo.z, lo.w), pack_bf16x2(hi.x, hi.y),
                          pack_bf16x2(hi.z, hi.w));
    } else {
        return reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.pool) + row * D)[c];
    }
}
template <int D, int M, typename Args>
__device__ __forceinline__ float pool_value(const Args& a, int64_t row, int e) {
    row += (int64_t)a.layer * a.num_pages * 2 * a.Hkv * a.P;
    if constexpr (e8<M>)
        return e4m3_values(static_cast<const uint8_t*>(a.pool)[row * D + e], __ldg(a.scales + row / kScaleRows)).x;
    else
        return __bfloat162float(static_cast<const __nv_bfloat16*>(a.pool)[row * D + e]);
}

// Whether some V row of the item is not finite; with a mask only of those that it
// hides.
template <int D, int M, typename Args>
__device__ bool has_odd_values(const Args& a, const BlockItem& it, const BlockRowMask* mask, int64_t values,
                               int lane) {
    const int per = pieces_of<M>(a), br = 128 / per;
    for (int j = it.t0; j < it.t0 + it.n_tiles; ++j) {
        const PrefillTile* t = a.tiles + j;
        const int2 r = __ldg(reinterpret_cast<const int2*>(t));
        const int key_b = __ldg(&t->key0b);
        if (mask && (r.y & kPrefillTileFull) && mask->whole(r.x) && mask->whole(key_b)) continue;
        for (int w = 0; w < 4; ++w) {
            const int key = (w < 2 ? r.x : key_b) + 32 * (w & 1) + lane;
            const uint32_t see = mask ? __ldg(&t->vis[w]) & mask->word(key - lane) : 0u;
            // (rows past the end were zeroed, a box that does not exist as well)
            const int page = __ldg(&a.tile_pages[(size_t)j * per + (w * 32 + lane) / br]);
            bool odd = false;
            if (!((see >> lane) & 1u) && page >= 0 && page < a.num_pages && key < it.n) {
                const int64_t v = values + (int64_t)page * 2 * a.Hkv * a.P + (key & (a.P - 1));
                for (int c = 0; c < D / 8; ++c) {
                    const uint4 x = pool_eight<D, M>(a, v, c);
                    const uint32_t xw[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        odd |= (xw[i] & 0x7f80u) == 0x7f80u || (xw[i] & 0x7f800000u) == 0x7f800000u;
                }
            }
            if (__any_sync(0xffffffffu, odd)) return true;
        }
    }
    return false;
}
template <int D, int M, typename Args>
__device__ __noinline__ void rows_again(const Args& a, const BlockItem& it, int tile, uint32_t rows, int row0,
                                        float m_run, float l, int lane) {
    constexpr int kCols = D / 32, kRows = 4, kAhead = 8;
    const int g = it.head & (kBlockTwoTiles - 1), per = pieces_of<M>(a), br = 128 / per;
    const int64_t keys = (int64_t)g * a.P, values = keys + (int64_t)a.Hkv * a.P;  // rows of page 0
    const bool odd = has_odd_values<D, M>(a, it, nullptr, values, lane);
    while (rows) {
        // up to kRows rows of one query: they see the same keys
        const int qi = tile * a.BP + (row0 + __ffs(rows) - 1) / a.G;
        int n_rows = 0, row[kRows];
        float m[kRows], inv[kRows], sum[kRows], acc[kRows][kCols];
        const uint4* q[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int next = row0 + __ffs(rows) - 1;
            const bool more = rows && tile * a.BP + next / a.G == qi;
            row[r] = more ? next : row[0];
            if (more) {
                rows &= rows - 1;
                ++n_rows;
            }
            m[r] = __shfl_sync(0xffffffffu, m_run, row[r] - row0);
            if (m[r] == -INFINITY) m[r] = 0.f;
            // (half of an average's weights: their own sum, taken below, may pass 1)
            const float l_row = __shfl_sync(0xffffffffu, l, row[r] - row0);
            inv[r] = l_row > 0.f ? 0.5f / l_row : 0.f;
            sum[r] = 0.f;
            q[r] = reinterpret_cast<const uint4*>(
                static_cast<const __nv_bfloat16*>(a.q) +
                ((size_t)(it.q_row + qi) * a.Hq + g * a.G + row[r] % a.G) * D);
#pragma unroll
            for (int i = 0; i < kCols; ++i) acc[r][i] = 0.f;
        }
        BlockRowMask mask;
        mask.init(a, it, qi);
        if (odd && !has_odd_values<D, M>(a, it, &mask, values, lane)) continue;
        for (int x = 0; x < 4 * it.n_tiles; ++x) {
            const int j = it.t0 + (x >> 2), w = x & 3;
            const PrefillTile* t = a.tiles + j;
            const int key = __ldg(w < 2 ? &t->key0 : &t->key0b) + 32 * (w & 1) + lane;
            const uint32_t see = __ldg(&t->vis[w]) & mask.word(key - lane);
            if (!see) continue;
            int64_t at = 0;  // of the key's row
            float p[kRows] = {};
            if ((see >> lane) & 1u) {
                // (a page outside the pool was flagged, and page 0 read)
                const int page = __ldg(&a.tile_pages[(size_t)j * per + (w * 32 + lane) / br]);
                at = (int64_t)((uint32_t)page < (uint32_t)a.num_pages ? page : 0) * 2 * a.Hkv * a.P +
                     (key & (a.P - 1));
#pragma unroll 4
                for (int c = 0; c < D / 8; ++c) {
                    const uint4 kk = pool_eight<D, M>(a, keys + at, c);
                    const uint32_t kw[4] = {kk.x, kk.y, kk.z, kk.w};
#pragma unroll
                    for (int r = 0; r < kRows; ++r) {
                        const uint4 qq = q[r][c];
                        const uint32_t qw[4] = {qq.x, qq.y, qq.z, qq.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            p[r] = fmaf(__uint_as_float(kw[i] << 16), __uint_as_float(qw[i] << 16), p[r]);
                            p[r] = fmaf(__uint_as_float(kw[i] & 0xffff0000u),
                                        __uint_as_float(qw[i] & 0xffff0000u), p[r]);
                        }
                    }
                }
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    p[r] = __bfloat162float(__float2bfloat16(ex2_ftz(fmaf(p[r], a.scale_log2, -m[r])))) * inv[r];
                    sum[r] += p[r];
                }
            }
            for (int c0 = 0; c0 < 32; c0 += kAhead) {
                float v[kAhead][kCols];
#pragma unroll
                for (int c = 0; c < kAhead; ++c) {
                    const int64_t from = values + __shfl_sync(0xffffffffu, at, c0 + c);
                    const bool seen = (see >> (c0 + c)) & 1u;
#pragma unroll
                    for (int i = 0; i < kCols; ++i) v[c][i] = seen ? pool_value<D, M>(a, from, lane + 32 * i) : 0.f;
                }
#pragma unroll
                for (int c = 0; c < kAhead; ++c)
#pragma unroll
                    for (int r = 0; r < kRows; ++r) {
                        const float pc = __shfl_sync(0xffffffffu, p[r], c0 + c);
#pragma unroll
                        for (int i = 0; i < kCols; ++i) acc[r][i] = fmaf(pc, v[c][i], acc[r][i]);
                    }
            }
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (r >= n_rows) break;
            float total = sum[r];
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) total += __shfl_xor_sync(0xffffffffu, total, off);
            const float scale = total > 0.f ? 1.f / total : 0.f;
            const size_t q_head = (size_t)(it.q_row + qi) * a.Hq + g * a.G + row[r] % a.G;
#pragma unroll
            for (int i = 0; i < kCols; ++i) {
                const float f = acc[r][i] * scale;
                const int col = lane + 32 * i;
                if (it.part >= 0)
                    a.part_o[(((size_t)it.part * kPrefillQTiles + tile) * kPrefillRows + row[r]) * D + col] = f;
                else if (a.out_f32)
                    static_cast<float*>(a.out)[q_head * D + col] = f;
                else
                    static_cast<__nv_bfloat16*>(a.out)[q_head * D + col] = __float2bfloat16(f);
            }
        }
    }
}

// What a softmax warp carries from item to item, in two words so that the
// loop over key tiles keeps its registers: the loads of the items before, and,
// as bits of `par`, the parities of the hand-offs to wait for next.  The item
// itself stays in its ring slot until the warp has written its output.
struct SoftmaxPhase {
    uint32_t ub, par;
};
constexpr uint32_t kParS = 1, kParO = 2, kParX = 4;  // S_t, O_t, dual-key exchange
constexpr uint32_t kParPV = 8;  // (three S buffers) items of three key tiles or more

// A V row whose key no query sees (a span's, or in an unused slot of a partial page)
// has the weight 0, and 0 times an infinity or NaN is NaN.  Rows that sq_append_kv
// wrote are taken to be finite; those that sq_extend added may never have been
// written.  So in the instances for sequences that have such rows (kHides) the softmax
// warps zero the hidden rows of a tile's V before they hand over the P that the
// tile's first PV waits for: tile a's, or in dual-key mode the tile's own, warp wq of
// the four the rows of word wq of the visibility.  V of the item's key tile j (its
// loads begin with number ub) is waited for; its load needs no P of this tile or of
// the one before.  (Rows past the end the producer has zeroed.)  In every instance
// this would cost 32,768 queries, 40% masked, 3.25 -> 3.30 ms by the code generated
// around it, and by a warp of its own that takes V over from the loads 3.43 ms.
template <int D, int M>
__device__ __forceinline__ bool zero_hidden_values(const Smem& sm, const PrefillTile* tile, int n, uint32_t ub,
                                                   int j, int T, bool dual, int wq, volatile int* abort_flag,
                                                   int lane) {
    using C = PreCfg<D, M>;
    static_assert(C::kSlots >= 5, "V's slot was last that of a tile at least two before");
    const uint32_t u = ub + (!dual ? 2 * j + 1 : j + 2 < T ? 2 * j + 2 : T + j);  // (see load_of)
    const int key = __ldg(wq < 2 ? &tile->key0 : &tile->key0b) + 32 * (wq & 1);
    const uint32_t hidden = ~__ldg(&tile->vis[wq]) & low_bits_through(n - 1 - key);
    if (!hidden) return true;
    if (!warp_wait(sm.bar<D, M>(C::kBarFull + u % C::kSlots), (u / C::kSlots) & 1, abort_flag)) return false;
    uint8_t* v = sm.ptr + C::kOffRing + u % C::kSlots * C::kSlotBytes + wq * 32 * 128;
    for (int i = lane; i < 32 * C::kColBlocks * 8; i += 32) {
        const int r = i >> 3 & 31;
        if ((hidden >> r) & 1u)
            *reinterpret_cast<uint4*>(v + (i >> 8) * C::kBlockBytes + r * 128 + (i & 7) * 16) =
                make_uint4(0, 0, 0, 0);
    }
    fence_proxy_async_smem();
    return true;
}

// Softmax warpgroup of query tile t (one row per thread) and its epilogue,
// for one item.  False: a wait ran out.
template <int D, int M, typename Args>
__device__ bool prefill_softmax(const Args& a, const Smem& sm, uint32_t tmem, int t,
                                uint32_t k, SoftmaxPhase& ph, volatile int* abort_flag, int warp,
                                int lane) {
    using C = PreCfg<D, M>;
    const int wq = warp & 3;
    const int row = wq * 32 + lane;
    const Item it = make_item<M>(a, item_read<D, M>(sm, k));
    const bool dual = it.dual;
    const int T_cta = it.T, t0 = it.t0;
    // dual-key mode: both tiles hold tile a's queries, tile t takes key tiles
    // t, t + 2, t + 4, ... of the CTA's range
    const int qi = it.pos_lo + (dual ? 0 : t) * a.BP + row / a.G;
    int n_q = a.n_q;
    if constexpr (of_blocks<M>) n_q = item_block<D, M>(sm, k).n_q;
    const bool valid = row < a.BP * a.G && qi < n_q;
    const int T = dual ? (T_cta + 1 - t) / 2 : T_cta;
    const int kstep = dual ? 2 : 1, kfirst = dual ? t : 0;
    float* xchg = reinterpret_cast<float*>(sm.ptr + C::kOffXchg);
    // (three S buffers) the buffer of this tile's j-th key tile and the parity of its
    // hand-overs go by the key tile's number in the CTA's life, ub / 2 before
    const uint32_t number0 = ph.ub / 2 + kfirst;
    auto number = [=](int j) { return number0 + kstep * j; };
    // A warp none of whose rows is a query only keeps the barrier count: it
    // waits for each S and signals its P without computing (its rows of P
    // and O are never read back).
    if (!__any_sync(0xffffffffu, valid)) {
        for (int j = 0; j < T; ++j) {
            if constexpr (hides<M>) {
                const PrefillTile* tile = a.tiles + t0 + kfirst + kstep * j;
                if ((t == 0 || dual) && !(__ldg(&tile->flags) & kPrefillTileFull) &&
                    !zero_hidden_values<D, M>(sm, tile, a.n, ph.ub, kfirst + kstep * j, T_cta, dual, wq,
                                              abort_flag, lane))
                    return false;
            }
            uint32_t buf = t, parity = ph.par & kParS;
            if constexpr (C::kBufs > 2) {
                buf = number(j) % 3;
                parity = (number(j) / 3) & 1;
            }
            if (!warp_wait(sm.bar<D, M>(C::kBarS + buf), parity, abort_flag)) return false;
            if (C::kBufs == 2) ph.par ^= kParS;
            tc_fence_before();
            mbar_arrive(sm.bar<D, M>(C::kBarP + buf));
        }
        if (T > 0) ph.par ^= kParO;
        if (C::kBufs > 2 && T_cta > 2) ph.par ^= kParPV;
        if (dual) {
            mbar_arrive(sm.bar<D, M>(t == 1 ? C::kBarX : C::kBarXFree));
            // (tile b's next P waits for tile a's reads also here)
            if (t == 1 && !warp_wait(sm.bar<D, M>(C::kBarXFree), (ph.par & kParX) != 0, abort_flag))
                return false;
            ph.par ^= kParX;
        }
        return true;
    }
    // rows that are no query (their results are never read) mask as the last
    // one does and stay out of the warp's votes, so that a tile with some does
    // not take the masked, twice-computed path (2.33 instead of 1.77 us a tile)
    RowMask<M> mask;
    if constexpr (of_blocks<M>) mask.init(a, item_block<D, M>(sm, k), valid ? qi : n_q - 1);
    else mask.init(a, valid ? qi : n_q - 1);
    const uint32_t tl = tmem + ((uint32_t)(wq * 32) << 16);
    uint32_t buf = t;
    uint32_t col_s = C::kColS + (uint32_t)t * kPrefillKeys;
    const uint32_t col_o = C::kColO + (uint32_t)t * C::kOStep;
    const float sc = a.scale_log2;  // > 0 (the host raises a zero scale to a tiny one)
    // most that a row's weights of one tile may sum to without a look at their
    // maximum (a power of two above the running one).  A warp with rows that are
    // no query raises its maxima where a weight passes 2^8, as such warps did
    // when every tile of theirs took the path with the maximum: the largest
    // weight of a row is then more often exactly 1, and not rounded (with 2^16
    // the log-sum-exp of 3 queries over 9,892 tokens was off by 2.4e-5 instead
    // of 1.3e-5 of its size).
    //
    // A block of queries has few key tiles, often the sinks' few keys first, whose
    // maxima the window's raise: there a row starts at a maximum of 0 and a tile's
    // weights are accepted while its sum stays below 2^80 (and above 2^-40 where
    // they are the row's first), since a weight rounded to bf16 keeps its 8 bits at
    // any size and sums are fp32 (those that overflow: rows_again).  16,384 queries at
    // a window of 1,024 with 4 sinks: 367 -> 254 us, half of it the maxima of first
    // tiles.  To raise a maximum holds a CTA up for about 5 us, many more than its
    // instructions take: they are seldom run and come from memory.  With 2^40, which
    // each of 32 rows passes at a tile of its own where logits are large (deviations
    // of 10 and more), 8 trees of 16 over 8,001 .. 32,000 tokens took 113 us (now 94),
    // a prompt of 8,191 queries 430 (370).
    constexpr float kLeast = 0x1p-40f;
    const float accept = of_blocks<M> ? 0x1p80f : __all_sync(0xffffffffu, valid) ? 65536.f : 256.f;
    float m_run = of_blocks<M> ? 0.f : -INFINITY, l = 0.f;
    // {first keys, flags} of the next key tile; its visibility bits are read
    // only where a tile is masked (they would hold eight registers of the loop)
    const PrefillTile* tp = a.tiles + t0 + kfirst;
    int2 nk = make_int2(0, 0);
    int nb = 0;
    if (T > 0) {
        nk = __ldg(reinterpret_cast<const int2*>(tp));
        nb = __ldg(&tp->key0b);
    }
    for (int j = 0; j < T; ++j) {
        // this tile's record; the next one is fetched while this tile is worked on
        const int2 wk = nk;
        const int wb_ = nb;
        if (j + 1 < T) {
            nk = __ldg(reinterpret_cast<const int2*>(tp + kstep));
            nb = __ldg(&tp[kstep].key0b);
        }
        if constexpr (hides<M>) {
            if ((t == 0 || dual) && !(wk.y & kPrefillTileFull) &&
                !zero_hidden_values<D, M>(sm, tp, a.n, ph.ub, kfirst + kstep * j, T_cta, dual, wq, abort_flag,
                                          lane))
                return false;
        }
        uint32_t parity = ph.par & kParS;
        if constexpr (C::kBufs > 2) {
            buf = number(j) % 3;
            col_s = C::col_s(buf);
            parity = (number(j) / 3) & 1;
        }
        if (!warp_wait(sm.bar<D, M>(C::kBarS + buf), parity, abort_flag)) return false;
        if (C::kBufs == 2) ph.par ^= kParS;
        tc_fence_after();
        // Raw logits q.k (the scale is applied inside the exponent; it is > 0),
        // taken 64 columns at a time to keep registers low: one pass for the
        // row maximum, one for the weights.
        const bool unmasked = (wk.y & kPrefillTileFull) && mask.whole(wk.x) && mask.whole(wb_);
        // (a block's window masks many tiles of which every key exists: no load)
        auto exists = [&](int ww) {
            return of_blocks<M> && (wk.y & kPrefillTileFull) ? 0xffffffffu : __ldg(&tp->vis[ww]);
        };
        // Weights 2^(s * scale - m) with the running maximum m, two arguments
        // at a time with a packed FMA, rounded to bf16 into wt (32 words per
        // 64 keys).  The normaliser sums the same rounded weights that the PV
        // product takes (eight fp32 chains), so the output is a convex
        // combination of the V rows whatever the rounding.
        // Nothing is stored: S stays intact until the weights are accepted.
        const uint64_t sc2 = f2pack(sc, sc);
        uint32_t wt[2][32];
        uint32_t seen = unmasked ? 1u : 0u;  // (blocks) the row sees some key of the tile
        auto weights = [&](float m, float& tile_sum) {
            const float nmu = m == -INFINITY ? 0.f : -m;
            const uint64_t nmu2 = f2pack(nmu, nmu);
            float ls[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                uint32_t x[64];
                tmem_ld32(tl + col_s + 64 * hh, *reinterpret_cast<uint32_t(*)[32]>(&x[0]));
                tmem_ld32(tl + col_s + 64 * hh + 32, *reinterpret_cast<uint32_t(*)[32]>(&x[32]));
                tmem_wait_ld();
                if (!unmasked) {
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        const int ww = 2 * hh + w;
                        const uint32_t mw =
                            exists(ww) & mask.word((ww < 2 ? wk.x : wb_) + 32 * (ww & 1));
                        if constexpr (of_blocks<M>) seen |= mw;
#pragma unroll
                        for (int c = 0; c < 32; ++c)
                            if (!((mw >> c) & 1u)) x[32 * w + c] = 0xff800000u;  // -inf
                    }
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    const float x0 = __uint_as_float(x[2 * i]), x1 = __uint_as_float(x[2 * i + 1]);
                    float a0, a1;
                    f2unpack(ffma2(f2pack(x0, x1), sc2, nmu2), a0, a1);
                    const __nv_bfloat162 hb = __floats2bfloat162_rn(ex2_ftz(a0), ex2_ftz(a1));
                    wt[hh][i] = *reinterpret_cast<const uint32_t*>(&hb);
                    add_bf16x2_f32(wt[hh][i], ls[2 * (i & 3)], ls[2 * (i & 3) + 1]);
                }
            }
            tile_sum = ((ls[0] + ls[1]) + (ls[2] + ls[3])) + ((ls[4] + ls[5]) + (ls[6] + ls[7]));
        };
        // The maximum is raised lazily, so most tiles keep it: take the
        // weights with the current maximum and accept them when no row's sum
        // exceeds `accept`, which bounds every weight; no maximum is needed for
        // that.  Otherwise (or when a row has seen no key yet) find the tile's
        // maximum and redo the tile with it wherever it exceeds the running
        // one by more than 2^8.
        float mt = -INFINITY, tsum = 0.f;
        bool done = false;
        if constexpr (of_blocks<M>) {
            weights(m_run, tsum);
            done = !__any_sync(0xffffffffu,
                               valid && (tsum > accept || (l == 0.f && seen && tsum < kLeast)));
        } else if (__all_sync(0xffffffffu, m_run != -INFINITY || !valid)) {
            weights(m_run, tsum);
            done = !__any_sync(0xffffffffu, valid && tsum > accept);
        }
        if (!done) {
            // row maximum: three-input max over four independent chains
            float mx[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) mx[c] = -INFINITY;
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                uint32_t x[64];
                tmem_ld32(tl + col_s + 64 * hh, *reinterpret_cast<uint32_t(*)[32]>(&x[0]));
                tmem_ld32(tl + col_s + 64 * hh + 32, *reinterpret_cast<uint32_t(*)[32]>(&x[32]));
                tmem_wait_ld();
                if (!unmasked) {
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        const int ww = 2 * hh + w;
                        const uint32_t mw =
                            exists(ww) & mask.word((ww < 2 ? wk.x : wb_) + 32 * (ww & 1));
#pragma unroll
                        for (int c = 0; c < 32; ++c)
                            if (!((mw >> c) & 1u)) x[32 * w + c] = 0xff800000u;  // -inf
                    }
                }
#pragma unroll
                for (int c = 0; c < 64; c += 8) {
                    mx[0] = fmax3(mx[0], __uint_as_float(x[c]), __uint_as_float(x[c + 1]));
                    mx[1] = fmax3(mx[1], __uint_as_float(x[c + 2]), __uint_as_float(x[c + 3]));
                    mx[2] = fmax3(mx[2], __uint_as_float(x[c + 4]), __uint_as_float(x[c + 5]));
                    mx[3] = fmax3(mx[3], __uint_as_float(x[c + 6]), __uint_as_float(x[c + 7]));
                }
            }
            mt = fmaxf(fmax3(mx[0], mx[1], mx[2]), mx[3]) * sc;
        }
        if (done) {
            l += tsum;
        } else {
            // (a block's row without weights yet may also come down)
            const bool need = valid && (mt > m_run + 8.f || (of_blocks<M> && l == 0.f && seen && mt < m_run - 8.f));
            float alpha = 1.f;
            if (need) {
                alpha = of_blocks<M> && l == 0.f ? 1.f : exp2f(m_run - mt);
                m_run = mt;
                l *= alpha;
            }
            if (j > 0 && __any_sync(0xffffffffu, need)) {
                // O_t holds the products up to key tile j - 1 (complete: S_t(j)
                // was issued after them; with three buffers before the last, which
                // is waited for: the next needs this row's P): rescale it in place
                if constexpr (C::kBufs > 2) {
                    const int u = number(j) + 1;  // its QK was issued after that PV
                    const bool more = kfirst + kstep * j + 1 < T_cta;
                    if (!warp_wait(sm.bar<D, M>(more ? C::kBarS + u % 3 : C::kBarPV),
                                   more ? u / 3 & 1 : (ph.par & kParPV) != 0, abort_flag))
                        return false;
                    tc_fence_after();
                }
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32];
                    tmem_ld32(tl + col_o + c * 32, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                    tmem_st32(tl + col_o + c * 32, o);
                }
            }
            weights(m_run, tsum);
            l += tsum;
        }
        // P_t over the first half of S_t: keys 64 hh .. +63 to columns 32 hh .. +31.
        // One warp also sees that the tiles of the products that follow have
        // landed (long ago, as a rule): V_j, and the K tile of the next S.
        bool landed = true;
        uint32_t fv = 0, fk = 0, pv = 0, pk = 0;
        if (C::kBufs > 2 && wq == 0) {
            // (V_jj and K_{jj+3}, in the order of load_of)
            const int jj = kfirst + kstep * j;
            const bool more = jj + 3 < T_cta;
            const uint32_t uv = ph.ub + (more ? 2 * jj + 3 : T_cta + jj), uk = more ? uv + 1 : uv;
            fv = sm.bar<D, M>(C::kBarFull + uv % C::kSlots);
            pv = (uv / C::kSlots) & 1;
            fk = sm.bar<D, M>(C::kBarFull + uk % C::kSlots);
            pk = (uk / C::kSlots) & 1;
            landed = mbar_try_wait(fv, pv) & mbar_try_wait(fk, pk);
        } else if (wq == 0 && t == 0 && !dual) {
            const uint32_t uv = ph.ub + 2 * j + 1, uk = uv + 1;
            fv = sm.bar<D, M>(C::kBarFull + uv % C::kSlots);
            pv = (uv / C::kSlots) & 1;
            fk = j + 1 < T ? sm.bar<D, M>(C::kBarFull + uk % C::kSlots) : fv;
            pk = j + 1 < T ? (uk / C::kSlots) & 1 : pv;
            landed = mbar_try_wait(fv, pv) & mbar_try_wait(fk, pk);
        }
        tmem_st32(tl + col_s, wt[0]);
        tmem_st32(tl + col_s + 32, wt[1]);
        tmem_wait_st();
        if (!__all_sync(0xffffffffu, landed)) {
            if (!warp_wait(fv, pv, abort_flag) || !warp_wait(fk, pk, abort_flag)) return false;
        }
        tc_fence_before();
        mbar_arrive(sm.bar<D, M>(C::kBarP + buf));
        tp += kstep;
    }
    if (T > 0) {
        if (!warp_wait(sm.bar<D, M>(C::kBarO + t), (ph.par & kParO) != 0, abort_flag)) return false;
        ph.par ^= kParO;
    }
    if (C::kBufs > 2 && T_cta > 2) ph.par ^= kParPV;
    if (of_blocks<M> && l == 0.f) m_run = -INFINITY;  // no key seen
    // dual-key mode: tile b hands its (max, normaliser) to tile a, which
    // merges the two partial results of each row (weights 2^(m_t - max)) and
    // reads O_b, complete by tile b's wait above
    float wa = 1.f, wb = 0.f;
    tc_fence_after();
    if (dual && t == 1) {
        xchg[2 * row] = m_run;
        xchg[2 * row + 1] = l;
        tc_fence_before();
        mbar_arrive(sm.bar<D, M>(C::kBarX));
        // tile b's next P (and with it the products that overwrite O_b) waits
        // until tile a has read O_b
        if (!warp_wait(sm.bar<D, M>(C::kBarXFree), (ph.par & kParX) != 0, abort_flag)) return false;
        ph.par ^= kParX;
        tc_fence_after();
        return true;
    }
    if (dual) {
        if (!warp_wait(sm.bar<D, M>(C::kBarX), (ph.par & kParX) != 0, abort_flag)) return false;
        ph.par ^= kParX;
        tc_fence_after();
        const float mb = xchg[2 * row], lb = xchg[2 * row + 1];
        const float m_top = fmaxf(m_run, mb);
        wa = m_run == -INFINITY ? 0.f : exp2f(m_run - m_top);
        wb = mb == -INFINITY ? 0.f : exp2f(mb - m_top);
        l = l * wa + lb * wb;
        m_run = m_top;
    }
    // the item again, from its slot
    const Item end = make_item<M>(a, item_read<D, M>(sm, k));
    int q_row = end.pos_lo;
    if constexpr (of_blocks<M>) q_row = item_block<D, M>(sm, k).q_row;
    const bool again = prefill_write<D, M>(a, end, q_row, tl, col_o, t, row, valid, m_run, l, wa, wb);
    if (dual) {
        tc_fence_before();
        mbar_arrive(sm.bar<D, M>(C::kBarXFree));
    }
    if constexpr (of_blocks<M>) {
        const uint32_t rows = __ballot_sync(0xffffffffu, again && l < INFINITY);
        __syncwarp();  // the pairs' stores come before those of rows_again
        if (rows) rows_again<D, M>(a, item_block<D, M>(sm, k), t, rows, wq * 32, m_run, l, lane);
    }
    return true;
}

template <typename Args>
struct ModeOf;
template <>
struct ModeOf<PrefillArgs> : std::integral_constant<int, 0> {};
template <>
struct ModeOf<PrefillShortArgs> : std::integral_constant<int, kOneTile> {};
template <>
struct ModeOf<PrefillHideArgs> : std::integral_constant<int, kHides> {};
template <>
struct ModeOf<PrefillHideShortArgs> : std::integral_constant<int, kHides | kOneTile> {};
template <>
struct ModeOf<BlockArgs> : std::integral_constant<int, kBlocks> {};
template <>
struct ModeOf<BlockShortArgs> : std::integral_constant<int, kBlocks | kOneTile> {};
template <>
struct ModeOf<BlockArgs2> : std::integral_constant<int, kBlocks | kTwoProducers> {};
template <>
struct ModeOf<BlockShortArgs2> : std::integral_constant<int, kBlocks | kOneTile | kTwoProducers> {};
template <>
struct ModeOf<BlockShortKv8Args> : std::integral_constant<int, kE8 | kBlocks | kOneTile> {};
template <>
struct ModeOf<BlockShortKv8Args2> : std::integral_constant<int, kE8 | kBlocks | kOneTile | kTwoProducers> {};

template <int D, typename Args>
__global__ void __launch_bounds__(PreCfg<D, ModeOf<Args>::value>::kThreads, 1)
    sq_prefill_kernel(const __grid_constant__ CUtensorMap pool_map,
                      const __grid_constant__ CUtensorMap qmap, const Args a) {
    constexpr int M = ModeOf<Args>::value;
    using C = PreCfg<D, M>;
    extern __shared__ uint8_t smem_raw[];
    Smem sm;
    sm.ptr = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                        ~static_cast<uintptr_t>(1023));
    sm.base = smem_addr(sm.ptr);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm.ptr + C::kOffMisc);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(sm.ptr + C::kOffMisc + 4);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // The warp's role by the numbers above.  Rows in 8 bits: the softmax warps come
    // first (two whole warpgroups, which take registers that the others give up: 640
    // threads start with 96 each), then producer, issuer, second producer and a warp
    // without a role, then two warpgroups of converters.
    const int role = !e8<M> ? warp : warp < 8 ? warp + 2 : warp < 10 ? warp - 8 : warp;
    // the split-merging kernel that follows may be scheduled from here on
    grid_launch_dependents();
    if (role == 0 && lane == 0) {
        mbar_init(sm.bar<D, M>(C::kBarQ), 1);
        for (int s = 0; s < C::kSlots; ++s) {
            mbar_init(sm.bar<D, M>(C::kBarFull + s), e8<M> ? kConverters / kConvertGroups : 1);
            if (e8<M>) mbar_init(sm.bar<D, M>(C::kBarRaw + s), a.n_pieces > 2 ? 1 + C::kTileScales : 1);
            mbar_init(sm.bar<D, M>(C::kBarEmpty + s), 1);
        }
        for (int b = 0; b < C::kBufs; ++b) {
            mbar_init(sm.bar<D, M>(C::kBarS + b), 1);
            mbar_init(sm.bar<D, M>(C::kBarP + b), 128);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(sm.bar<D, M>(C::kBarO + b), 1);
        }
        if (C::kBufs > 2) mbar_init(sm.bar<D, M>(C::kBarPV), 1);
        mbar_init(sm.bar<D, M>(C::kBarVfix), 1);
        mbar_init(sm.bar<D, M>(C::kBarQFree), 1);
        mbar_init(sm.bar<D, M>(C::kBarDone), 1);
        for (int s = 0; s < kItemSlots; ++s) {
            mbar_init(sm.bar<D, M>(C::kBarItem + s), 1);
            mbar_init(sm.bar<D, M>(C::kBarItemFree + s), kItemReaders + producers<M> - 1 + (e8<M> ? kConverters : 0));
        }
        mbar_init(sm.bar<D, M>(C::kBarClc), 1);
        mbar_init(sm.bar<D, M>(C::kBarX), 128);
        mbar_init(sm.bar<D, M>(C::kBarXFree), 128);
        fence_mbar_init();
        *abort_flag = 0;
    }
    if (role == 1) {
        tmem_alloc(smem_addr(tmem_slot), C::kTmemCols);
        tmem_relinquish();
    }
    FirstItem<D, M> start;
    int u_early = 0;
    const bool second = producers<M> > 1 && role == kProducer2;  // the second producer warp
    if (role == 0 || second) {
        if (role == 0 && lane == 0) {
            prefetch_tmap(&pool_map);
            prefetch_tmap(&qmap);
        }
        if (a.plan_ready) start.read(a, second, lane);
        if constexpr (one_tile<M> && !e8<M>) {
            if (a.kv_early && role == 0) {
                const Item it = make_item<M>(a, start.item.raw);
                u_early = early_loads<D, M>(&pool_map, a, sm, start, it, lane);
            }
        }
    }
    // Launched as a programmatic dependent: the set-up above overlapped the
    // preceding kernel's tail; the queries and the pool, and a plan that was
    // not on the device before that kernel, are read only from here on (but for
    // the first K/V tiles of early_loads).
    grid_dependency_wait();
    if (role == 0 || second) {
        if (!a.plan_ready) start.read(a, second, lane);
        if (role == 0 && lane == 0) {  // the thread that initialised the barriers
            start.item.write(sm.ptr + C::kOffItems);
            mbar_arrive(sm.bar<D, M>(C::kBarItem));
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    // (a warpgroup's registers change at the head of its roles' branch)
    if (e8<M> && warp >= 12) {
        if constexpr (e8<M>) {
            take_registers<C::kConvertRegs, false>();
            convert_tiles<D, M>(sm, a.err, abort_flag, warp - 12, lane);
        }
    } else if (e8<M> && warp >= 8) {
        if constexpr (e8<M>) {
            take_registers<C::kOtherRegs, false>();
            if (role == 0 || second)
                block_produce<D, M>(&pool_map, &qmap, a, sm, start, u_early, abort_flag, second, lane);
            else if (role == 1 && lane == 0)
                prefill_mma<D, M>(a, sm, tmem, abort_flag);
            __syncwarp();
        }
    } else if (role == 0) {
        if constexpr (of_blocks<M>)
            block_produce<D, M>(&pool_map, &qmap, a, sm, start, u_early, abort_flag, 0, lane);
        else
            prefill_produce<D, M>(&pool_map, &qmap, a, sm, start, u_early, abort_flag, lane);
    } else if (second) {
        if constexpr (of_blocks<M>)
            block_produce<D, M>(&pool_map, &qmap, a, sm, start, u_early, abort_flag, 1, lane);
    } else if (role == 1) {
        if (lane == 0) prefill_mma<D, M>(a, sm, tmem, abort_flag);
        __syncwarp();
    } else {
        if constexpr (e8<M>) take_registers<C::kSoftmaxRegs, true>();
        const int t = (role - 2) >> 2;
        SoftmaxPhase ph = {0, 0};
        bool ok;
        for (uint32_t k = 0;; ++k) {
            ok = __all_sync(0xffffffffu, item_wait<D, M>(sm, k, abort_flag));
            if (!ok) break;
            const int4 raw = item_read<D, M>(sm, k);
            if (raw.z < 0) break;
            const Item it = make_item<M>(a, raw);
            if (t == 0 || it.two || it.dual) {
                ok = prefill_softmax<D, M>(a, sm, tmem, t, k, ph, abort_flag, warp, lane);
                if (!ok) break;
            }
            ph.ub += 2 * raw.z;
            __syncwarp();
            if (lane == 0) item_free<D, M>(sm, k);
        }
        if (!ok && lane == 0) {
            if (!*abort_flag) set_error(a.err, kErrTimeout);
            *abort_flag = 1;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (role == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, C::kTmemCols);
    }
}

// Merges the key-range splits of each query row: weights 2^(lse_s - max).
// One warp per (split unit, row, 32 V columns); the lanes take the splits' log-
// sum-exps (up to 64 splits).  The partial outputs of the first U splits are
// loaded together with them, so a row of up to U splits costs one round trip;
// an empty split's partial (never written) is read but selected away.  The
// kernel lets the next one be scheduled at once: a next layer's prefill CTAs
// take the SMs as this layer's leave.
//
// What bounds it: the loads in flight.  Many rows of few splits (a split last
// round: 10,240 rows of 7) want many warps, each with a whole row in few
// registers (V = D / 32, U = 8); few rows of many splits (an 8-query call: 256
// rows of 19) one round trip, spread over the SMs (V = 2, U = 24).  With the
// second form for both, a turn with four layers of the former took 2,500 us
// instead of 2,484; with the first for both, an 8-query call needs three round
// trips for its 19 splits.
constexpr int kCombineThreads = 128;
constexpr int kCombineFew = 8;  // splits up to which the first form is used
template <int D, int V, int U, typename Args>  // V: output elements per lane, U: splits per batch of loads
__global__ void __launch_bounds__(kCombineThreads, U > kCombineFew ? 6 : 8)
    sq_prefill_combine_kernel(const Args a) {
    constexpr bool kOfBlocks = std::is_same<Args, BlockCombineArgs>::value;
    constexpr int kParts = D / (32 * V);
    grid_launch_dependents();
    const int gw = (int)((blockIdx.x * blockDim.x + threadIdx.x) >> 5);
    const int lane = threadIdx.x & 31;
    constexpr int kRowsPerUnit = kPrefillQTiles * kPrefillRows;
    const int m = gw / (a.rows * kParts);
    if (m >= a.n_merges) return;
    const int tr = (gw / kParts) % a.rows, col = (gw % kParts) * 32 * V + lane * V;
    // the plan was uploaded before the prefill kernel started
    const auto mg = a.merges[m];
    const int n_split = mg.n;
    const int t = tr / kPrefillRows, row = tr % kPrefillRows;
    // the row's KV head and query, and the end of the queries
    int g, qi, n_q;
    if constexpr (kOfBlocks) {
        g = mg.g;
        qi = mg.q_row + t * a.BP + row / a.G;
        n_q = mg.q_row + mg.n_q;
    } else {
        const int qt = mg.unit / a.Hkv;
        g = mg.unit % a.Hkv;
        qi = (qt * kPrefillQTiles + t) * a.BP + row / a.G;
        n_q = a.n_q;
    }
    // programmatic dependent of the prefill kernel: wait for its partials
    grid_dependency_wait();
    if (row >= a.BP * a.G || qi >= n_q) return;
    const int h = g * a.G + row % a.G;
    // partial row of split s: part0 + s * kRowsPerUnit
    const size_t part0 = ((size_t)mg.part0 * kPrefillQTiles + t) * kPrefillRows + row;
    const float ml0 = lane < n_split ? a.part_ml[part0 + (size_t)lane * kRowsPerUnit] : -INFINITY;
    const float ml1 =
        lane + 32 < n_split ? a.part_ml[part0 + (size_t)(lane + 32) * kRowsPerUnit] : -INFINITY;
    float vals[U][V];
    auto load = [&](int s0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + u;  // the same in every lane
            const float* po = a.part_o + (part0 + (size_t)s * kRowsPerUnit) * D + col;
#pragma unroll
            for (int e = 0; e < V; ++e) vals[u][e] = 0.f;
            if (s >= n_split) continue;
            if constexpr (V == 4) {
                const float4 v = *reinterpret_cast<const float4*>(po);
                vals[u][0] = v.x; vals[u][1] = v.y; vals[u][2] = v.z; vals[u][3] = v.w;
            } else {
                const float2 v = *reinterpret_cast<const float2*>(po);
                vals[u][0] = v.x; vals[u][1] = v.y;
            }
        }
    };
    load(0);
    float M = fmaxf(ml0, ml1);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
    float w0 = 0.f, w1 = 0.f;
    if (M != -INFINITY) {
        if (ml0 != -INFINITY) w0 = exp2f(ml0 - M);
        if (ml1 != -INFINITY) w1 = exp2f(ml1 - M);
    }
    float W = w0 + w1;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) W += __shfl_xor_sync(0xffffffffu, W, off);
    float none = 0.f;  // of a row without weights; NaN where a piece's are NaN
    if (__any_sync(0xffffffffu, ml0 != ml0 || ml1 != ml1)) W = none = NAN;
    float inv = W > 0.f ? 1.f / W : none;
    const float lse = W > 0.f ? (M + __log2f(W)) * 0.69314718055994531f : none - INFINITY;
    // (blocks: an average at every step, so that the largest values do not overflow)
    if (kOfBlocks && W > 0.f) {
        w0 *= inv;
        w1 *= inv;
        inv = 1.f;
    }
    float acc[V] = {};
    for (int s0 = 0; W > 0.f && s0 < n_split; s0 += U) {
        if (s0 > 0) load(s0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + u;
            const float ws = __shfl_sync(0xffffffffu, s < 32 ? w0 : w1, s & 31);
            if (s < n_split && ws > 0.f) {
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += ws * vals[u][e];
            }
        }
    }
    const size_t o = ((size_t)qi * a.Hq + h) * D + col;
    if (a.out_f32) {
        float* out = reinterpret_cast<float*>(a.out) + o;
        if constexpr (V == 4)
            *reinterpret_cast<float4*>(out) =
                make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
        else
            *reinterpret_cast<float2*>(out) = make_float2(acc[0] * inv, acc[1] * inv);
    } else {
        __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(a.out) + o;
        if constexpr (V == 4) {
            uint2 u;
            u.x = pack_bf16x2(acc[0] * inv, acc[1] * inv);
            u.y = pack_bf16x2(acc[2] * inv, acc[3] * inv);
            *reinterpret_cast<uint2*>(out) = u;
        } else {
            *reinterpret_cast<uint32_t*>(out) = pack_bf16x2(acc[0] * inv, acc[1] * inv);
        }
    }
    if (lane == 0 && col == 0 && a.lse) a.lse[(size_t)qi * a.Hq + h] = lse;
}

}  // namespace
}  // namespace dev

}  // namespace sq
