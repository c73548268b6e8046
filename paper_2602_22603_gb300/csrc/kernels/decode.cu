// Split-K flash-decoding over the paged bf16 KV pool, with the log-sum-exp
// merge of its partial results in the same kernel.
//
// What is computed (Sec. 1 and Sec. 3.4: for every generated token,
// attention reads the whole KV cache of the context; Sec. 2.1: in
// grouped-query attention a K/V head serves G query heads): for sequence i,
// query head h and KV head g = h / G,
//     out[i][h] = sum_t softmax_t(sm_scale * q[i][h] . K_g[t]) V_g[t].
//
// Work decomposition (host planner, core.cpp): every run of pages that a
// group of sequences holds in common (a main thread and its forked auxiliary
// threads, Sec. 3.4) is one segment; a (segment, KV head) pair is a list of
// 64-token stages; the stages of all pairs are dealt evenly to persistent
// CTAs, one per SM.
//
// A CTA has two consumer groups of four warps, each with a producer warp and a
// TMA + mbarrier ring of its own (2 x 96 KiB in flight per SM); the groups take
// alternate stages.  A consumer warp owns 16 tokens of a stage and keeps an
// online-softmax partial (max, sum, unnormalised output) for up to 16 query
// rows - the G heads of every sequence in the segment's group, so a shared page
// is read from HBM once for all of them.  At an item's end the consumers leave
// their rows in shared memory and go on; two closing warps add them, write the
// item's partial and merge what it completes.
//
// What bounds it: HBM in long calls (the read probe's rate at 128k); in short
// ones the chain after the last stage (add, partial, arrival, merge: 5 us from
// the slowest CTA's last stage to the next call's start) and the SMs' unequal
// shares of HBM (2 us between most and the slowest).  Two CTAs per SM with the
// same ring space, each closing its items itself, left twice the entries per
// run and stalled at every item's end.  Per call at 32q/8kv, d = 128, so and
// now: one sequence of 32,768 tokens 27.5 and 24.6 us, 36 sequences of 250 ..
// 6,000 tokens 51.4 and 46.4 us, four agents and their forks at 20,000 ..
// 60,000 tokens with partial pages 54.6 and 45.6 us; eight of 131,072 and their
// forks 600 us either way.  Prefetching stages past the ring into L2 while the
// previous call ends gains nothing: 6 instead of 4 stages 795 -> 810 us for 32
// layers of the 32k sequence.
//
// Merge: an item leaves one partial (max, sum, unnormalised output) per group
// member, in that (sequence, KV head)'s contiguous run of entries; a member
// whose run is this one item gets its normalised output directly.  After an
// item a CTA counts its arrival on each of the item's runs; the CTA that brings
// a count to the number of entries merges that run (max of the maxima, weights
// 2^(m - M)) and writes the normalised output.  Counts are zero in every
// uploaded plan and the merger resets its count, so every call starts from
// zero.
//
// Start-up: the kernel is a programmatic dependent of whatever precedes it.
// When the plan was already on the device (a reused plan), every role reads its
// first items before the dependency wait, and stages in pages that no running
// work writes are loaded before it.
//
// Windows (single tokens of sq_window_attention): a sequence's pages are then the
// sinks' and the window's, the rows before the window's first masked the way a
// page's unused slots are.
//
// Page fills: after a ragged eviction a page may hold fewer rows than it has
// slots (its rows first; what the others hold is masked).  Stages are in
// slot space (page index x P + slot); the plan then carries every page's
// fill, and the rows past a page's fill get no weight.
//
// Tensor cores: S = Q K^T and O += P V are m16n8k16 bf16 mma.sync with fp32
// accumulation; rows = query rows (<= 16), columns = tokens / head dims.  The
// contraction is tiny (G x d per token) and the kernel is HBM-bound, so the
// warp-level mma is the right size: the point is to keep HBM busy.
#include <math.h>

#include <type_traits>

#include "e4m3.cuh"
#include "launch.hpp"
#include "ptx.cuh"

namespace sq {
namespace {

using namespace dev;

// kE8: rows in 8 bits (see kv8.hpp).
template <bool kE8>
using ArgsOf = std::conditional_t<kE8, DecodeKv8Args, DecodeArgs>;
template <int D, bool kE8>
struct DecCfg {
    static constexpr int kColBlocks = kE8 ? 1 : D / 64;          // column blocks of a row
    static constexpr int kRowBytes = kE8 ? D : 128;              // ... and a row's bytes in one
    static constexpr int kBlockBytes = kStageTokens * kRowBytes; // one column block of a tile
    static constexpr int kTileBytes = kColBlocks * kBlockBytes;  // K (or V) of one stage
    static constexpr int kStageBytes = 2 * kTileBytes;
    // per group: 96 KiB in flight (80 where rows are 128 bytes)
    static constexpr int kStages = kE8 ? (D == 128 ? 5 : 12) : (D == 128 ? 3 : 6);
    static constexpr int kConsumers = kDecodeConsumerWarps * 32;
    static constexpr int kRingBytes = kDecodeGroups * kStages * kStageBytes;
    // warps: consumers, a producer per group, two that close items
    static constexpr int kClosers = 64;
    static constexpr int kThreads = kConsumers + kDecodeGroups * 32 + kClosers;
    static constexpr int kOffBars = kRingBytes;
    // barriers: per group full [kStages], empty [kStages]; then the three of the
    // items' ends; then the abort flag
    static constexpr int kBarOut = kDecodeGroups * 2 * kStages;  // a pass's rows are written
    static constexpr int kBarOutFree = kBarOut + 1;              // ... and read
    static constexpr int kBarRuns = kBarOut + 2;                 // the last item's runs are listed
    static constexpr int kBarBytes = kE8 ? 512 : 256;
    // (8 bits) a stage's scales: its blocks' of keys, then of values
    static constexpr int kStageScales = kE8 ? 2 * kStageTokens / kScaleRows : 0;
    static constexpr int kOffScales = kOffBars + kBarBytes;
    static constexpr int kOffRed = kOffScales + kDecodeGroups * kStages * kStageScales * 4;
    // item ends: per-warp row max / sum, eight rows of every warp's output, and
    // the runs an item completed
    static constexpr int kPassRows = 8;
    static constexpr int kOffRuns = kOffRed + 2 * kDecodeConsumerWarps * kRowsPerTile * 4;
    static constexpr int kOffOut = kOffRuns + 256;
    static constexpr int kOutBytes = kDecodeConsumerWarps * kPassRows * D * 4;
    static constexpr int kSmemBytes = kOffOut + kOutBytes + 1024;  // + alignment slack
    // (bf16 rows) 8-wide output column tiles, 16-deep contraction steps
    static constexpr int kNT = D / 8;
    static constexpr int kKS = D / 16;
    static_assert(kSmemBytes <= 232448 && kOffOut % 16 == 0, "shared memory");
    static_assert((kBarRuns + 1) * 8 + 4 <= kBarBytes, "mbarriers");
    static_assert(kOffScales % 16 == 0 && kOffRed % 16 == 0, "alignment");
};

__device__ __forceinline__ uint32_t ld_u32(const __nv_bfloat16* p) {
    return *reinterpret_cast<const uint32_t*>(p);
}

// Sum of the two bf16 halves of a packed pair, in fp32.
__device__ __forceinline__ float bf16x2_sum(uint32_t v) {
    return __uint_as_float(v << 16) + __uint_as_float(v & 0xffff0000u);
}

// ---- producers: one warp per group issues the TMA loads of its stages --------
// The groups take alternate stages of the CTA, each through a ring of its own.
// The warp walks its stages in order; the page of the next stage is read while
// the current one waits for its slot.  Whole-page stages (P >= 64) are issued by
// lane 0; with smaller pages each lane issues one box (page, column block, K or
// V).
template <int D>
struct Producer {
    using C = DecCfg<D, false>;
    const CUtensorMap* tmap;
    const DecodeArgs& a;
    uint8_t* ring;      // the group's slots
    uint64_t* bars;     // the group's barriers: full [kStages], empty [kStages]
    volatile int* abort_flag;
    int group, lane;
    // this lane's box within a stage of small pages
    int box_page, box_cb, box_kv;
    // the current stage: stage s of item it (it0 .. it1), and its lane's page
    int it, it1, s, s1, head, page_off, n_pages;
    int32_t pid;      // -1: no box for this lane
    int slot;
    uint32_t phase;   // parity of the slot's use
    uint32_t issued, issued_phase;  // per-slot bits of the last issue
    bool first;       // the CTA's first stage has not gone out yet

    __device__ void init() {
        box_cb = lane % C::kColBlocks;
        box_kv = (lane / C::kColBlocks) % 2;
        box_page = a.P < kStageTokens ? lane / (2 * C::kColBlocks) : 0;
        it = a.cta_begin[blockIdx.x];
        it1 = a.cta_begin[blockIdx.x + 1];
        slot = 0;
        phase = 0;
        issued = issued_phase = 0;
        first = group == 0;
        if (it < it1) {
            open_item();
            s += group;
            settle();
        }
    }
    __device__ bool more() const { return it < it1; }
    __device__ void open_item() {
        const DecodeItem* item = a.items + it;
        const DecodeSeg* seg = a.segs + item->seg;
        s = item->s0;
        s1 = item->s1;
        head = item->head;
        page_off = seg->page_off;
        n_pages = seg->n_pages;
    }
    // Carries a stage past the item's end into the items that follow.
    __device__ void settle() {
        while (s >= s1) {
            const int over = s - s1;
            if (++it == it1) return;
            open_item();
            s += over;
        }
        const int pi = s * kStageTokens / a.P + box_page;
        const int per = a.P < kStageTokens ? kStageTokens / a.P : 1;
        pid = box_page < per && pi < n_pages ? a.page_ids[page_off + pi] : -1;
    }
    __device__ int row(int kv) const {
        const int row0 = a.P > kStageTokens ? (s * kStageTokens) & (a.P - 1) : 0;
        return (kv ? a.Hkv + head : head) * a.P + row0;
    }
    __device__ void advance() {
        first = false;
        if (++slot == C::kStages) {
            slot = 0;
            phase ^= 1;
        }
        s += kDecodeGroups;
        settle();
    }
    // Issues the current stage into its (free) slot.
    __device__ void issue() {
        const uint32_t full = smem_addr(&bars[slot]);
        const uint32_t dst = smem_addr(ring) + slot * C::kStageBytes;
        if (a.P >= kStageTokens) {
            if (lane == 0) {
                if ((uint32_t)pid < (uint32_t)a.num_pages) {
                    mbar_arrive_expect_tx(full, C::kStageBytes);
                    const int rk = row(0), rv = row(1);
#pragma unroll
                    for (int cb = 0; cb < C::kColBlocks; ++cb) {
                        tma_load_4d(dst + cb * C::kBlockBytes, tmap, full, cb * 64, rk, pid, a.layer);
                        tma_load_4d(dst + cb * C::kBlockBytes + C::kTileBytes, tmap, full, cb * 64, rv,
                                    pid, a.layer);
                    }
                } else {
                    set_error(a.err, kErrBounds);
                    mbar_arrive(full);
                }
            }
        } else {
            const bool valid = pid >= 0 && pid < a.num_pages;
            if (pid < -1 || pid >= a.num_pages) set_error(a.err, kErrBounds);
            const uint32_t n = __popc(__ballot_sync(0xffffffffu, valid));
            if (lane == 0) {
                if (n) mbar_arrive_expect_tx(full, n * a.P * 128u);
                else mbar_arrive(full);
            }
            __syncwarp();
            if (valid)
                tma_load_4d(dst + box_kv * C::kTileBytes + box_cb * C::kBlockBytes +
                                box_page * a.P * 128,
                            tmap, full, box_cb * 64, row(box_kv), pid, a.layer);
        }
        issued |= 1u << slot;
        issued_phase = (issued_phase & ~(1u << slot)) | (phase << slot);
    }
    // Before the grid-dependency wait (a plan that was on the device): stages in
    // pages that no running work writes are loaded, up to the ring's depth, and
    // the first few of the others prefetched into L2.
    __device__ void early() {
        if ((int)blockIdx.x == a.debug_drop_cta) return;
        int n = 0;
        if (a.kv_early && a.P >= kStageTokens) {
            for (; n < C::kStages && more(); ++n) {
                bool unsafe = false;
                for (int u = lane; u < a.n_unsafe; u += 32) unsafe |= a.unsafe[u] == pid;
                if (__any_sync(0xffffffffu, unsafe)) break;
                issue();
                advance();
            }
        }
        // (the walk goes on from here after the wait: look ahead on a copy)
        Producer ahead = *this;
        for (; n < kPrefetchStages && ahead.more(); ++n) {
            if (ahead.pid >= 0 && ahead.pid < a.num_pages && (a.P < kStageTokens || lane < 2 * C::kColBlocks))
                tma_prefetch_l2_4d(tmap, box_cb * 64, ahead.row(box_kv), ahead.pid, a.layer);
            ahead.advance();
        }
    }
    static constexpr int kPrefetchStages = 4;
    __device__ void run() {
        bool ok = true;
        while (more()) {
            const uint32_t empty = smem_addr(&bars[C::kStages + slot]);
            ok = __all_sync(0xffffffffu, mbar_wait(empty, phase ^ 1, abort_flag));
            if (!ok) break;
            // test hook: leave this stage unsignalled (the consumers' bounded wait
            // runs out; nothing is in flight for it)
            if (!(first && (int)blockIdx.x == a.debug_drop_cta)) issue();
            advance();
        }
        if (!ok && lane == 0) {
            if (!*abort_flag) set_error(a.err, kErrTimeout);
            *abort_flag = 1;
            // Leave only after every copy already issued has landed (bounded).
            for (int sl = 0; sl < C::kStages; ++sl)
                if ((issued >> sl) & 1u)
                    mbar_wait(smem_addr(&bars[sl]), (issued_phase >> sl) & 1u);
        }
        __syncwarp();
    }
};

// The same for rows in 8 bits, whose stages pass twice as fast: what the producer did
// for each held them up (1,470 of 1,690 cycles a stage, with the consumers waiting 600 of
// theirs).  So it walks the plan a batch of an item's stages at a time, a lane to each
// stage's page (each of its pages, where it has several), and reads an item's record two
// items ahead and its segment's one item: 48 sequences of 200 .. 60,000 tokens take 160
// us of 156 for their bytes at 128 dimensions, and at 64 on pages of 16 120 (then 116;
// stage by stage, page ids read four stages ahead, 194).  With a second batch's page ids
// read in advance they took 121: the walk past an item's end waits for its loads sooner.
//
// A box has the rows of a page (64 at most) of keys and of values, one after the other,
// since every box costs its thread about 100 cycles (windows of 2,048 tokens of 64
// sequences on pages of 16: 18.9 -> 17.1 us).  The lane that issues it also copies the
// page's scales: in bulk (kWhole, pages of 64 tokens or more: 32 bytes of either plane),
// else by cp.async (a bulk copy takes no less than 16 bytes).
template <int D, bool kWhole>
struct ProducerE8 {
    using C = DecCfg<D, true>;
    static constexpr int kHalf = C::kStageScales / 2;
    static constexpr int kMost = D == 128 ? 4 : 8;   // stages of a batch
    static constexpr int kEarly = 4;                 // stages that may go out before the wait
    static_assert(kMost <= C::kStages && kEarly <= C::kStages, "slots that are free at the start");
    // The next stages of one item: their KV head, and of the lane's the first row in its
    // page and the page, -1: none.
    struct Batch {
        int n, head, row;
        int32_t pid;
    };
    struct Item {
        int s0, s1, head, seg, page_off, n_pages;
    };
    const CUtensorMap* tmap;
    const DecodeKv8Args& a;
    uint32_t ring;      // the group's slots (shared address)
    uint32_t scales;    // ... and their scales
    uint32_t bars;      // ... and barriers: full [kStages], empty [kStages]
    volatile int* abort_flag;
    int group, lane;
    int log_q, stage, part;      // (pages of a stage: 1 << log_q) the lane's of a batch
    int most;                    // stages of a batch
    int it, it1, s, log_p;       // the walk: stage s of item `it`
    Item cur, nx, n2;            // the item, the next one, and the one after without its segment
    int64_t page_scales;         // scales of a page, all planes
    const float* layer_scales;
    Batch w;
    int slot;
    uint32_t phase, issued;
    bool first;                  // the CTA's first stage has not gone out yet

    __device__ __forceinline__ void init() {
        log_p = __ffs(a.P) - 1;
        log_q = kWhole ? 0 : __ffs(kStageTokens) - 1 - log_p;
        stage = lane >> log_q;
        part = lane & ((1 << log_q) - 1);
        most = min(kMost, 32 >> log_q);
        page_scales = (int64_t)2 * a.Hkv * (a.P / kScaleRows);
        layer_scales = a.scales + (int64_t)a.layer * a.num_pages * page_scales;
        it = a.cta_begin[blockIdx.x];
        it1 = a.cta_begin[blockIdx.x + 1];
        slot = 0;
        phase = issued = 0;
        first = group == 0;
        read_item(it, cur);
        read_item(it + 1, nx);
        read_item(it + 2, n2);
        read_segment(cur);
        read_segment(nx);
        s = cur.s0 + group;
        next();
    }
    __device__ __forceinline__ void read_item(int i, Item& x) const {
        const DecodeItem* item = a.items + (i < it1 ? i : 0);
        x.s0 = item->s0;
        x.s1 = item->s1;
        x.head = item->head;
        x.seg = item->seg;
    }
    __device__ __forceinline__ void read_segment(Item& x) const {
        x.page_off = a.segs[x.seg].page_off;
        x.n_pages = a.segs[x.seg].n_pages;
    }
    // Carries the walk past an item's end into the items that follow.
    __device__ __forceinline__ void settle() {
        while (it < it1 && s >= cur.s1) {
            s += nx.s0 - cur.s1;
            ++it;
            cur = nx;
            nx = n2;
            read_segment(nx);
            read_item(it + 2, n2);
        }
    }
    // The walk's next stages of its item, and on behind them.
    __device__ __forceinline__ void next() {
        static_assert(kDecodeGroups == 2, "a group's stages are every other one");
        settle();
        w.n = it < it1 ? min(most, (cur.s1 - s + 1) >> 1) : 0;
        w.head = cur.head;
        const int st = s + 2 * stage;
        w.row = kWhole ? (st * kStageTokens) & (a.P - 1) : 0;
        const int at = ((st * kStageTokens) >> log_p) + part;
        w.pid = stage < w.n && at < cur.n_pages ? a.page_ids[cur.page_off + at] : -1;
        s += 2 * w.n;
    }
    // Issues the batch's stage j into the (free) slot.
    __device__ __forceinline__ void issue(int j) {
        if (stage == j) {
            const uint32_t full = bars + 8 * slot;
            const uint32_t dst = ring + slot * C::kStageBytes, sdst = scales + slot * C::kStageScales * 4;
            const bool valid = w.pid >= 0 && w.pid < a.num_pages;
            if (w.pid < -1 || w.pid >= a.num_pages) set_error(a.err, kErrBounds);
            const float* src = layer_scales + w.pid * page_scales + w.head * (a.P / kScaleRows);
            if constexpr (kWhole) {
                if (valid) {
                    src += w.row / kScaleRows;
                    mbar_arrive_expect_tx(full, C::kStageBytes + C::kStageScales * 4);
                    load_pair(dst, full);
                    bulk_load(sdst, src, kHalf * 4, full);
                    bulk_load(sdst + kHalf * 4, src + page_scales / 2, kHalf * 4, full);
                } else {
                    mbar_arrive(full);
                }
            } else {
                if (valid) {
                    mbar_arrive_expect_tx(full, a.P * 2 * C::kRowBytes);
                    load_pair(dst + part * a.P * 2 * C::kRowBytes, full);
                    const uint32_t to = sdst + part * (a.P / kScaleRows) * 4;
                    copy_scales(to, src);
                    copy_scales(to + kHalf * 4, src + page_scales / 2);
                } else {
                    mbar_arrive(full);
                }
                // (arrives when this lane's copies have landed)
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(full) : "memory");
            }
        }
        __syncwarp();
    }
    // A page's scales of one plane and head: 1, 2 or 4.
    __device__ __forceinline__ void copy_scales(uint32_t dst, const float* src) const {
        if (a.P == 8)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
        else if (a.P == 16)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
        else
            asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    }
    // A page's box of keys and of values.
    __device__ __forceinline__ void load_pair(uint32_t dst, uint32_t full) const {
        asm volatile(
            "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
            " [%0], [%1, {%3, %4, %5, %6, %7}], [%2];" ::"r"(dst),
            "l"(tmap), "r"(full), "r"(0), "r"(w.row), "r"(w.head), "r"(0), "r"(a.layer * a.num_pages + w.pid)
            : "memory");
    }
    __device__ __forceinline__ void next_slot() {
        first = false;
        ++issued;
        if (++slot == C::kStages) {
            slot = 0;
            phase ^= 1;
        }
    }
    // Before the grid-dependency wait (see Producer): of the first batch's first kEarly
    // stages those in pages that no running work writes; the others are prefetched into
    // L2.  Returns the stages issued.
    __device__ __forceinline__ int early() {
        if ((int)blockIdx.x == a.debug_drop_cta) return 0;
        int n = 0;
        bool go = kWhole && a.kv_early;
        for (int j = 0; j < min(w.n, kEarly); ++j) {
            const int32_t pid = __shfl_sync(0xffffffffu, w.pid, j);
            bool unsafe = false;
            for (int u = lane; u < a.n_unsafe; u += 32) unsafe |= a.unsafe[u] == pid;
            go = go && !__any_sync(0xffffffffu, unsafe);
            if (go) {
                issue(j);
                next_slot();
                ++n;
            } else if (stage == j && w.pid >= 0 && w.pid < a.num_pages) {
                asm volatile("cp.async.bulk.prefetch.tensor.5d.L2.global.tile [%0, {%1, %2, %3, %4, %5}];" ::"l"(tmap),
                             "r"(0), "r"(w.row), "r"(w.head), "r"(0), "r"(a.layer * a.num_pages + w.pid)
                             : "memory");
            }
        }
        return n;
    }
    // n: stages of the first batch that went out early.
    __device__ __forceinline__ void run(int n) {
        bool ok = true;
        while (ok && w.n > 0) {
            for (int j = 0; j < w.n; ++j) {
                if (j < n) continue;
                ok = __all_sync(0xffffffffu, mbar_wait(bars + 8 * (C::kStages + slot), phase ^ 1, abort_flag));
                if (!ok) break;
                // test hook: leave this stage unsignalled (see Producer)
                if (!(first && (int)blockIdx.x == a.debug_drop_cta)) issue(j);
                next_slot();
            }
            n = 0;
            next();
        }
        if (!ok && lane == 0) {
            if (!*abort_flag) set_error(a.err, kErrTimeout);
            *abort_flag = 1;
            // Leave only after every copy already issued has landed (bounded; a stage that
            // the test hook left out is waited for in vain).
            for (uint32_t u = issued > C::kStages ? issued - C::kStages : 0; u < issued; ++u)
                mbar_wait(bars + 8 * (u % C::kStages), (u / C::kStages) & 1);
        }
        __syncwarp();
    }
    // The producer warp's whole life.
    __device__ __forceinline__ void live() {
        int n = 0;
        if (a.plan_ready) init();
        named_bar_sync(2, C::kThreads);  // (the barriers are initialised)
        if (a.plan_ready) n = early();
        grid_dependency_wait();
        grid_launch_dependents();
        if (!a.plan_ready) init();
        run(n);
    }
};

// ---- consumers: two groups of four warps, 16 tokens of a stage per warp ------
// The groups take alternate stages of the CTA.  Every consumer warp runs every
// item and reaches every named barrier of every item, also after a wait ran
// out (it then skips the work only), so the barriers never miss a participant.

// What a consumer lane needs of an item before its first stage; read one item
// ahead.  (The token count and the members' limits are not among it: an append
// may rewrite them in a plan that is on the device, so they are read after the
// dependency wait.)
struct ItemHead {
    int seg, head, s0, s1, n_grp, seq0, seq1;
    __device__ void read(const DecodeArgs& a, int it, int j0, int j1) {
        const DecodeItem* item = a.items + it;
        seg = item->seg;
        head = item->head;
        s0 = item->s0;
        s1 = item->s1;
        const DecodeSeg* sg = a.segs + seg;
        n_grp = sg->n_grp;
        seq0 = sg->grp_seq[j0];  // (entries past n_grp are zero)
        seq1 = sg->grp_seq[j1];
    }
};

// One fp32 row of the item-end merge: eight-float blocks XORed with the row, so
// that the eight rows of a warp's store hit different banks.
template <int D>
__device__ __forceinline__ int out_pos(int row, int col) {
    return row * D + ((((col >> 3) ^ row) & (D / 8 - 1)) << 3) + (col & 7);
}

// Four consecutive output elements from element `at`: v * inv.
__device__ __forceinline__ void write_out(const DecodeArgs& a, size_t at, const float4& v, float inv) {
    if (a.out_f32) {
        *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + at) =
            make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
    } else {
        uint2 u;
        u.x = pack_bf16x2(v.x * inv, v.y * inv);
        u.y = pack_bf16x2(v.z * inv, v.w * inv);
        *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(a.out) + at) = u;
    }
}

// Adds the consumer warps' rows rb .. rb + 7 of an item (weights 2^(m_w - M),
// warps in order) and writes its partials or outputs: `n` threads, `v0` = which.
template <int D, bool kE8>
__device__ __forceinline__ void close_rows(const DecodeArgs& a, const DecodeItem* item,
                                           const DecodeSeg* seg, int head, int sole, int rows, int rb,
                                           const uint8_t* smem, int v0, int n) {
    using C = DecCfg<D, kE8>;
    constexpr int kVec = D / 4;  // float4 per output row
    const int G = a.G;
    const float* red_m = reinterpret_cast<const float*>(smem + C::kOffRed);
    const float* red_l = red_m + kDecodeConsumerWarps * kRowsPerTile;
    const float* red_o = reinterpret_cast<const float*>(smem + C::kOffOut);
    const int n_out = min(rows - rb, (int)C::kPassRows) * kVec;
    for (int v = v0; v < n_out; v += n) {
        const int pr = v / kVec, c4 = v % kVec, r = rb + pr, j = r / G;
        // a member whose run is this item alone gets its normalised output
        const bool alone = (sole >> j) & 1;
        const int to = alone ? seg->grp_seq[j] : item->ent[j];
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < kDecodeConsumerWarps; ++w) M = fmaxf(M, red_m[w * kRowsPerTile + r]);
        const float Ms = M == -INFINITY ? 0.f : M;
        float L = 0.f;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kDecodeConsumerWarps; ++w) {
            const float f = exp2f(red_m[w * kRowsPerTile + r] - Ms);
            L += red_l[w * kRowsPerTile + r] * f;
            const float4 x =
                *reinterpret_cast<const float4*>(red_o + w * C::kPassRows * D + out_pos<D>(pr, c4 * 4));
            sum.x += x.x * f; sum.y += x.y * f; sum.z += x.z * f; sum.w += x.w * f;
        }
        if (alone) {
            write_out(a, ((size_t)to * a.Hq + head * G + r % G) * D + c4 * 4, sum, 1.f / L);
        } else {
            const size_t pe = (size_t)to * G + r % G;
            *reinterpret_cast<float4*>(a.part_o + pe * D + c4 * 4) = sum;
            if (c4 == 0)
                *reinterpret_cast<float4*>(a.part_ml + pe * 4) = make_float4(M, L, 0.f, 0.f);
        }
    }
}

template <int D>
__device__ void consume(const DecodeArgs& a, int it0, int it1, ItemHead next, uint8_t* smem,
                        uint64_t* all_bars, volatile int* abort_flag, int warp, int lane) {
    using C = DecCfg<D, false>;
    const int gid = lane >> 2, tig = lane & 3;
    const int r0 = gid, r1 = gid + 8;
    const int mi = lane >> 3, rr = lane & 7;
    const int group = warp >> 2, w4 = warp & 3;
    const int G = a.G;
    const int j0 = r0 / G, j1 = r1 / G;
    uint64_t* bars = all_bars + group * 2 * C::kStages;
    float* red_m = reinterpret_cast<float*>(smem + C::kOffRed);     // [8][16]
    float* red_l = red_m + kDecodeConsumerWarps * kRowsPerTile;     // [8][16]
    float* red_o = reinterpret_cast<float*>(smem + C::kOffOut);     // [8][8][D], out_pos
    uint32_t n_pass = 0;  // item-end passes so far
    uint8_t* ring = smem + group * C::kStages * C::kStageBytes;  // the group's slots
    int slot = 0;
    uint32_t phase = 0;
    int skip = group;   // stages to the group's next one
    bool dead = false;  // warp-uniform: a wait ran out or the CTA aborted
    for (int it = it0; it < it1; ++it) {
        const ItemHead item = next;
        const DecodeSeg* seg = a.segs + item.seg;
        const int n_grp = item.n_grp;
        const bool v0 = j0 < n_grp, v1 = j1 < n_grp;
        const int lim0 = v0 ? seg->grp_lim[j0] : 0;
        const int lim1 = v1 ? seg->grp_lim[j1] : 0;
        const int n_tok = seg->n_tok;

        uint32_t qa[C::kKS][4];
        {
            const __nv_bfloat16* q0 =
                a.q + ((size_t)(v0 ? item.seq0 : 0) * a.Hq + item.head * G + r0 % G) * D;
            const __nv_bfloat16* q1 =
                a.q + ((size_t)(v1 ? item.seq1 : 0) * a.Hq + item.head * G + r1 % G) * D;
#pragma unroll
            for (int kk = 0; kk < C::kKS; ++kk) {
                const int c = kk * 16 + tig * 2;
                qa[kk][0] = v0 ? ld_u32(q0 + c) : 0u;
                qa[kk][1] = v1 ? ld_u32(q1 + c) : 0u;
                qa[kk][2] = v0 ? ld_u32(q0 + c + 8) : 0u;
                qa[kk][3] = v1 ? ld_u32(q1 + c + 8) : 0u;
            }
        }
        if (it + 1 < it1) next.read(a, it + 1, j0, j1);
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        float o[C::kNT][4];
#pragma unroll
        for (int nd = 0; nd < C::kNT; ++nd) o[nd][0] = o[nd][1] = o[nd][2] = o[nd][3] = 0.f;

        int s = item.s0 + skip;
        for (; s < item.s1; s += kDecodeGroups) {
            const uint32_t full = smem_addr(&bars[slot]);
            const uint32_t empty = smem_addr(&bars[C::kStages + slot]);
            // Pages a ragged eviction left partial: bit r of vm says whether
            // row r of this warp's 16 holds a row of its page (read before
            // the wait, off the critical path).  The others' scores are masked,
            // and their V rows zeroed before the product.
            uint32_t vm = 0xffffu;
            if (a.page_fill) {
                // P is a power of two >= 8 and the 16 rows start at a multiple
                // of 16: one page holds them all (P >= 16), or two (P = 8)
                const int P = a.P;
                const int t0 = s * kStageTokens + w4 * 16;  // segment slot position
                const int pq = t0 >> (__ffs(P) - 1);
                const int f0 = pq < seg->n_pages ? __ldg(&a.page_fill[seg->page_off + pq]) : 0;
                auto rows = [](int f, int from, int most) {
                    // the first rows up to x, of `most` from row `from` on
                    auto up_to = [&](int x) { return (1u << min(max(x - from, 0), most)) - 1u; };
                    return (up_to(f & kFillMask) & ~up_to(f >> kFillFirstBit & kFillMask)) |
                           up_to(f >> kFillSinkBit);
                };
                if (P >= 16) {
                    vm = rows(f0, t0 & (P - 1), 16);
                } else {
                    const int f1 =
                        pq + 1 < seg->n_pages ? __ldg(&a.page_fill[seg->page_off + pq + 1]) : 0;
                    vm = rows(f0, 0, 8) | rows(f1, 0, 8) << 8;
                }
            }
            if (!dead) {
                const bool ok = mbar_wait(full, phase, abort_flag);
                if (!__all_sync(0xffffffffu, ok)) {
                    if (lane == 0 && !*abort_flag) set_error(a.err, kErrTimeout);
                    *abort_flag = 1;
                    dead = true;
                }
            }
            if (!dead) {
                const uint32_t kb = smem_addr(ring + slot * C::kStageBytes);
                const uint32_t vb = kb + C::kTileBytes;
                const int tbase = s * kStageTokens + w4 * 16;  // segment-relative

                // S = Q K^T over this warp's 16 tokens (two n8 tiles)
                float sc[2][4];
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) sc[nt][0] = sc[nt][1] = sc[nt][2] = sc[nt][3] = 0.f;
                {
                    const int t = w4 * 16 + (mi >> 1) * 8 + rr;
                    const uint32_t row = kb + t * 128;
                    const int sw = t & 7;
#pragma unroll
                    for (int kk = 0; kk < C::kKS; ++kk) {
                        const int d0 = kk * 16 + (mi & 1) * 8;
                        uint32_t b0, b1, b2, b3;
                        ldsm_x4(row + (d0 >> 6) * C::kBlockBytes + ((((d0 & 63) >> 3) ^ sw) << 4), b0,
                                b1, b2, b3);
                        mma_bf16(sc[0], qa[kk], b0, b1);
                        mma_bf16(sc[1], qa[kk], b2, b3);
                    }
                }

                // masking, scaling, online softmax (log2 domain)
                float x[2][4];
                float mx0 = -INFINITY, mx1 = -INFINITY;
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int tk = tbase + nt * 8 + tig * 2 + e;
                        const bool rv = (vm >> (nt * 8 + tig * 2 + e)) & 1u;
                        x[nt][e] = tk < lim0 && rv ? sc[nt][e] * a.scale_log2 : -INFINITY;
                        x[nt][2 + e] = tk < lim1 && rv ? sc[nt][2 + e] * a.scale_log2 : -INFINITY;
                        mx0 = fmaxf(mx0, x[nt][e]);
                        mx1 = fmaxf(mx1, x[nt][2 + e]);
                    }
                mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 1));
                mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, 2));
                mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 1));
                mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, 2));
                const float mn0 = fmaxf(m0, mx0), mn1 = fmaxf(m1, mx1);
                const float ms0 = mn0 == -INFINITY ? 0.f : mn0;
                const float ms1 = mn1 == -INFINITY ? 0.f : mn1;
                const float al0 = exp2f(m0 - ms0), al1 = exp2f(m1 - ms1);
                m0 = mn0;
                m1 = mn1;
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        x[nt][e] = exp2f(x[nt][e] - ms0);
                        x[nt][2 + e] = exp2f(x[nt][2 + e] - ms1);
                    }
                // P in bf16 for the PV product; the normaliser sums the same
                // rounded weights, so the output is an exact convex combination
                uint32_t pa[4];
                pa[0] = pack_bf16x2(x[0][0], x[0][1]);
                pa[1] = pack_bf16x2(x[0][2], x[0][3]);
                pa[2] = pack_bf16x2(x[1][0], x[1][1]);
                pa[3] = pack_bf16x2(x[1][2], x[1][3]);
                const float ps0 = bf16x2_sum(pa[0]) + bf16x2_sum(pa[2]);
                const float ps1 = bf16x2_sum(pa[1]) + bf16x2_sum(pa[3]);
                l0 = l0 * al0 + ps0;
                l1 = l1 * al1 + ps1;
#pragma unroll
                for (int nd = 0; nd < C::kNT; ++nd) {
                    o[nd][0] *= al0;
                    o[nd][1] *= al0;
                    o[nd][2] *= al1;
                    o[nd][3] *= al1;
                }

                // Rows past the last valid token hold stale or never-written
                // shared memory, and rows that their page's fill hides may hold
                // anything: zero this warp's such V rows so 0 * V stays 0.
                const bool tail = tbase + 16 > n_tok || vm != 0xffffu;
                if (tail) {
                    const uint32_t live = vm & ((1u << min(max(n_tok - tbase, 0), 16)) - 1u);
                    constexpr int per_row = C::kColBlocks * 8;  // 16-byte chunks per row
                    uint8_t* vgen = ring + slot * C::kStageBytes + C::kTileBytes;
                    for (int idx = lane; idx < 16 * per_row; idx += 32) {
                        const int r = idx / per_row, rem = idx % per_row;
                        if (!((live >> r) & 1u))
                            *reinterpret_cast<uint4*>(vgen + (rem >> 3) * C::kBlockBytes + (w4 * 16 + r) * 128 +
                                                      (rem & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    __syncwarp();
                }

                // O += P V (V^T fragments through ldmatrix.trans)
                {
                    const int t = w4 * 16 + (mi & 1) * 8 + rr;
                    const uint32_t row = vb + t * 128;
                    const int sw = t & 7;
#pragma unroll
                    for (int nd2 = 0; nd2 < C::kKS; ++nd2) {
                        const int d0 = nd2 * 16 + (mi >> 1) * 8;
                        uint32_t b0, b1, b2, b3;
                        ldsm_x4_trans(row + (d0 >> 6) * C::kBlockBytes + ((((d0 & 63) >> 3) ^ sw) << 4),
                                      b0, b1, b2, b3);
                        mma_bf16(o[2 * nd2], pa, b0, b1);
                        mma_bf16(o[2 * nd2 + 1], pa, b2, b3);
                    }
                }
                if (tail) fence_proxy_async_smem();  // generic writes before the next TMA fill
                __syncwarp();
                if (lane == 0) mbar_arrive(empty);
            }
            if (++slot == C::kStages) {
                slot = 0;
                phase ^= 1;
            }
        }
        skip = s - item.s1;

        // Leave the item's rows to the closing warps, eight at a time, and go on
        // with the next item: nothing here waits for the other consumers.
        l0 += __shfl_xor_sync(0xffffffffu, l0, 1);
        l0 += __shfl_xor_sync(0xffffffffu, l0, 2);
        l1 += __shfl_xor_sync(0xffffffffu, l1, 1);
        l1 += __shfl_xor_sync(0xffffffffu, l1, 2);
        const int rows = n_grp * G;
        const bool last = it + 1 == it1;
        for (int rb = 0; rb < rows; rb += C::kPassRows, ++n_pass) {
            // the previous pass's rows have been read
            if (!dead && n_pass > 0 && !(last && rb > 0)) {
                const bool ok =
                    mbar_wait(smem_addr(&all_bars[C::kBarOutFree]), (n_pass - 1) & 1, abort_flag);
                if (!__all_sync(0xffffffffu, ok)) {
                    if (lane == 0 && !*abort_flag) set_error(a.err, kErrTimeout);
                    *abort_flag = 1;
                    dead = true;
                }
            }
            if (dead && !last) continue;
            const int r = rb + gid;  // this lane's row of the pass: r0, then r1
            if (tig == 0) {
                red_m[warp * kRowsPerTile + r] = rb ? m1 : m0;
                red_l[warp * kRowsPerTile + r] = rb ? l1 : l0;
            }
            if (r < rows) {
                float* wo = red_o + warp * C::kPassRows * D;
#pragma unroll
                for (int nd = 0; nd < C::kNT; ++nd)
                    *reinterpret_cast<float2*>(wo + out_pos<D>(gid, nd * 8 + tig * 2)) =
                        rb ? make_float2(o[nd][2], o[nd][3]) : make_float2(o[nd][0], o[nd][1]);
            }
            if (last) {
                // nothing is left to stream: the consumers add the rows themselves
                // (every warp gets here, also after a wait ran out)
                const int sole = a.items[it].sole;
                named_bar_sync(1, C::kConsumers);
                close_rows<D, false>(a, a.items + it, seg, item.head, sole, rows, rb, smem, threadIdx.x,
                              C::kConsumers);
                if (rb + C::kPassRows < rows) {
                    named_bar_sync(1, C::kConsumers);
                    continue;
                }
            }
            __syncwarp();
            if (lane == 0 && !dead) mbar_arrive(smem_addr(&all_bars[C::kBarOut]));
        }
    }
}

// ---- rows in 8 bits -------------------------------------------------------------
// The products take fp16: an e4m3 code is exact in it, and one conversion makes two.
// A power of two for each query row takes it from bf16 into fp16's range, the largest
// element to 2^14 .. 2^15 (elements below 2^-32 of it lose digits); the logits are
// taken back with the softmax's scale and their block's, one factor for the eight keys
// of a block, and, where that might be an infinity (and make NaN of a key of zeros), a
// power of two as the softmax takes them.
//
// The keys are the rows of the first product, S^T = K Q^T, and the values' dimensions
// those of the second, O^T = V^T P^T, so that the query rows are the columns, eight to a
// product: with one sequence of 4 or 8 heads a group none is wasted (when this was
// chosen, 16 sequences of 20,001 .. 60,000 tokens, 64/8 heads: 200.5 us with the query rows
// as the sixteen rows, 174.8 so, now 143; two stages of a warp at a time, whose chains
// overlap, gain nothing, nor do they at 64 dimensions: 114.9 and 112.9 us over 48 long
// contexts, 15.8 and 17.1 over 64 windows of 2,048, now 118.5 and 16.7).
// ldmatrix moves 16-bit pairs, here two neighbouring
// dimensions.  Keys: a lane gets dimensions 4 tig .. 4 tig + 3 of sixteen, so the
// queries' fragments are loaded in that order.  Values, transposed: the pairs of two
// tokens; the bytes are taken apart, the even dimensions being the first eight rows of
// a product and the odd ones the others.  P is transposed by movmatrix.
//
// Weights are w = 2^(x - m), m a reference that is raised only where some weight passes
// 2^kMost, to the largest logit less kLift.  The normaliser sums them rounded to fp16: 11
// digits down to 2^-14, an error of 2^-25 below, which is 2^-32 of the largest weight's.
// A block's values have their scale s, so what goes into the product is w s / v, v being
// a power of two of the row's own that is raised where some w s passes 2^kMost v, to at
// most 2^-kLift of it, and comes down as m goes up; rounded once, so that what a key adds
// is off by 2^-12 of itself, or by 2^-32 of what the row's largest w s stands for.  (One
// reference for all rows of a warp, the largest scale met, lost every value 2^25 below an
// outlier's, whatever the outlier's weight; 48 contexts of 200 .. 60,000 tokens, 32/8 heads
// of 128 dimensions, took 158.8 us and 160.4 so, 64/8 of 64 115 and 118.5, 64 windows of
// 2,048 15.9 and 16.7.)  The sums get v back at the item's end, and
// 2^-kMost with it (the normaliser too), so that they are of weights of at most 1: with
// weights of 2^kMost they pass what fp32 holds where values are large.
constexpr float kLift = 7.f, kMost = 15.f;
static_assert(kMost == 15.f, "0x7800 of a stage, 0x1p-15f at an item's end");
constexpr float kNoKeys = -3.4028234e38f;   // m at a row's start: no logit is below

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32"
        " {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t max_f16x2(uint32_t a, uint32_t b) {
    const __half2 v = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&v);
}
// a *= x, b *= y.
__device__ __forceinline__ void scale_pair(float& a, float& b, float x, float y) {
    asm("{\n\t.reg .b64 u, v;\n\tmov.b64 u, {%0, %1};\n\tmov.b64 v, {%2, %3};\n\t"
        "mul.rn.f32x2 u, u, v;\n\tmov.b64 {%0, %1}, u;\n\t}"
        : "+f"(a), "+f"(b)
        : "f"(x), "f"(y));
}
// Whether either half of a is above b's.
__device__ __forceinline__ bool above_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("{\n\t.reg .pred p, q;\n\tsetp.gt.f16x2 p|q, %1, %2;\n\tor.pred p, p, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(r)
        : "r"(a), "r"(b));
    return r != 0;
}
// lo += the low half of w, hi += its high half.
__device__ __forceinline__ void add_f16x2(uint32_t w, float& lo, float& hi) {
    asm("{\n\t.reg .b16 l16, h16;\n\tmov.b32 {l16, h16}, %2;\n\t"
        "add.rn.f32.f16 %0, l16, %0;\n\tadd.rn.f32.f16 %1, h16, %1;\n\t}"
        : "+f"(lo), "+f"(hi)
        : "r"(w));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t w) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(w));
    return r;
}

// Exponent of the power of two at or below a positive number (0: -127).
__device__ __forceinline__ int exponent_of(float x) { return (__float_as_int(x) >> 23) - 127; }

// A query row (head h of the call; one that is none is zero) as B fragments, and the
// two factors that its logits take: row gid of a column tile.
template <int D>
__device__ __forceinline__ float2 load_query_f16(const DecodeArgs& a, size_t h, bool on, int tig,
                                                uint32_t (&qb)[D / 16][2]) {
    uint32_t most = 0;
    const uint2* row = reinterpret_cast<const uint2*>(a.q + h * D) + tig;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
        const uint2 x = on ? row[kk * 4] : make_uint2(0u, 0u);
        qb[kk][0] = x.x;
        qb[kk][1] = x.y;
        // (sizes of bf16 order as their bits)
        most = max(max(most, x.x << 16 & 0x7fffffffu), x.x & 0x7fff0000u);
        most = max(max(most, x.y << 16 & 0x7fffffffu), x.y & 0x7fff0000u);
    }
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
    const int k = max((int)(most >> 23) - 127, -100) - 14;
    const float f = power_of_two(-k);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t x = qb[kk][e];
            qb[kk][e] = pack_f16x2(__uint_as_float(x << 16) * f, __uint_as_float(x & 0xffff0000u) * f);
        }
    // (a product that passes fp32: one key has all the weight with any such factor)
    const float c = fminf(a.scale_log2 * power_of_two(k), 3.4028234e38f);
    const int up = min(max(exponent_of(c), 0), 126);
    return make_float2(c * power_of_two(-up), power_of_two(up));
}

// The plan's entries of the pages that a warp's 16 tokens of a stage lie in (two where
// pages have 8), and which of the tokens hold rows of their pages, as in consume().
__device__ __forceinline__ int2 e8_fills(const DecodeArgs& a, int page_off, int n_pages, int tbase) {
    const int pq = tbase >> (__ffs(a.P) - 1);
    int2 f = make_int2(0, 0);
    if (pq < n_pages) f.x = __ldg(&a.page_fill[page_off + pq]);
    if (a.P == 8 && pq + 1 < n_pages) f.y = __ldg(&a.page_fill[page_off + pq + 1]);
    return f;
}
__device__ __forceinline__ uint32_t e8_rows(int f, int from, int most) {
    // the first rows up to x, of `most` from row `from` on
    auto up_to = [&](int x) { return (1u << min(max(x - from, 0), most)) - 1u; };
    return (up_to(f & kFillMask) & ~up_to(f >> kFillFirstBit & kFillMask)) | up_to(f >> kFillSinkBit);
}
__device__ __forceinline__ uint32_t e8_filled(int2 fills, int P, int tbase) {
    return P >= 16 ? e8_rows(fills.x, tbase & (P - 1), 16) : e8_rows(fills.x, 0, 8) | e8_rows(fills.y, 0, 8) << 8;
}

// What a consumer warp carries through an item: NR column tiles of eight query rows.
template <int D, int NR>
struct E8State {
    uint32_t qb[NR][D / 16][2];
    float o[D / 16][NR][4];   // dimensions 16 j + 2 gid (+ 1), rows 2 tig, 2 tig + 1
    float c[NR][2], up[NR][2];   // what logits take: below 4, and a power of two, 1 or more
    float m[NR][2], l[NR][2];
    float iv[NR][2];          // 1 / v
};

// A stage's 16 tokens of a warp, in the ring's slot at `tile` (shared address), which
// has the scales `sc`.  kAll: every row sees every token; else row (r, e) those of bits
// see[r][e], and `live` says which tokens are the segment's.
template <int D, int NR, bool kAll>
__device__ __forceinline__ void e8_stage(E8State<D, NR>& st, uint8_t* tile, const float* sc, uint32_t live,
                                         const uint32_t (&see)[NR][2], int box_rows, int w4, int lane) {
    using C = DecCfg<D, true>;
    const int gid = lane >> 2, mi = lane >> 3, rr = lane & 7;
    // (this lane's row of a matrix, in a box's keys or, `box_rows` further, values; the
    // swizzle's turn and the matrix's half of a step)
    const int t = w4 * 16 + (mi & 1) * 8 + rr;
    auto key_row = [&](int row) { return 2 * row - (row & (box_rows - 1)); };
    const uint32_t at = smem_addr(tile) + key_row(t) * D, turn = (mi >> 1) ^ (D == 128 ? t & 7 : t >> 1 & 3);
    float2 sk = *reinterpret_cast<const float2*>(sc + w4 * 2);
    float2 sv = *reinterpret_cast<const float2*>(sc + C::kStageScales / 2 + w4 * 2);
    if (!kAll) {
        // a block without rows of the segment has no scale worth reading
        if (!(live & 0xffu)) sk.x = 0.f, sv.x = power_of_two(kLeastScale);
        if (!(live >> 8)) sk.y = 0.f, sv.y = power_of_two(kLeastScale);
    }
    // logits
    float x[NR][4];
    {
        float acc[NR][2][4] = {};   // (even and odd steps apart, where there is one tile)
#pragma unroll
        for (int k2 = 0; k2 < D / 32; ++k2) {
            // tokens 0 .. 7 and 8 .. 15 of an even step, then of the odd one
            uint32_t b[4];
            ldsm_x4(at + ((turn ^ (2 * k2)) << 4), b[0], b[1], b[2], b[3]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t f[4] = {e4m3_to_f16x2(b[2 * h]), e4m3_to_f16x2(b[2 * h + 1]),
                                       e4m3_to_f16x2(b[2 * h] >> 16), e4m3_to_f16x2(b[2 * h + 1] >> 16)};
#pragma unroll
                for (int r = 0; r < NR; ++r)
                    mma_f16(acc[r][NR > 1 ? 0 : h], f, st.qb[r][2 * k2 + h][0], st.qb[r][2 * k2 + h][1]);
            }
        }
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float f0 = st.c[r][e] * sk.x, f1 = st.c[r][e] * sk.y;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    float s = acc[r][0][2 * b + e];
                    if (NR == 1) s += acc[r][1][2 * b + e];
                    s *= b ? f1 : f0;
                    if (!kAll && !(see[r][e] >> (gid + 8 * b) & 1u)) s = -INFINITY;
                    x[r][2 * b + e] = s;
                }
            }
    }
    // weights, and what goes into the second product (w s first: it passes fp32's range
    // only where some reference has to be raised)
    uint32_t h[NR][2], p[NR][2], pb[NR][2];
    auto weigh = [&] {
#pragma unroll
        for (int r = 0; r < NR; ++r)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const float w0 = exp2f(fmaf(x[r][2 * b], st.up[r][0], -st.m[r][0]));
                const float w1 = exp2f(fmaf(x[r][2 * b + 1], st.up[r][1], -st.m[r][1])), s = b ? sv.y : sv.x;
                h[r][b] = pack_f16x2(w0, w1);
                p[r][b] = pack_f16x2(w0 * s * st.iv[r][0], w1 * s * st.iv[r][1]);
            }
    };
    weigh();
    uint32_t most = 0;
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int b = 0; b < 2; ++b) most = max_f16x2(most, max_f16x2(h[r][b], p[r][b]));
    if (__any_sync(0xffffffffu, above_f16x2(most, 0x78007800u))) {  // (2^kMost)
        // references from the largest logits, and from the largest w s
        auto largest = [](float y) {
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, off));
            return y;
        };
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            float f[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                // (of either block: its largest w s is its largest logit's)
                const float x0 = largest(x[r][e]) * st.up[r][e], x1 = largest(x[r][2 + e]) * st.up[r][e];
                const float m = fmaxf(st.m[r][e], fmaxf(x0, x1) - kLift);
                const float al = exp2f(st.m[r][e] - m);
                st.m[r][e] = m;
                st.l[r][e] *= al;
                const float ws = fmaxf(exp2f(x0 - m) * sv.x, exp2f(x1 - m) * sv.y);
                const int v0 = -exponent_of(st.iv[r][e]);
                const int v = min(max(max(v0 + exponent_of(al), exponent_of(ws) - (int)kLift), -126), 126);
                st.iv[r][e] = power_of_two(-v);
                f[e] = al * power_of_two(max(v0 - v, -126));
            }
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                scale_pair(st.o[j][r][0], st.o[j][r][1], f[0], f[1]);
                scale_pair(st.o[j][r][2], st.o[j][r][3], f[0], f[1]);
            }
        }
        weigh();
    }
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            pb[r][b] = transpose_8x8(p[r][b]);
            add_f16x2(h[r][b], st.l[r][0], st.l[r][1]);
        }
    if (!kAll) {
        // V rows that hold none of the segment's may hold anything: zero them, so that
        // 0 * V stays 0
        for (int i = lane; i < D; i += 32) {   // 16-byte chunks of 16 rows
            const int r = i / (D / 16);
            if (!((live >> r) & 1u))
                *reinterpret_cast<uint4*>(tile + (key_row(w4 * 16 + r) + box_rows) * D + i % (D / 16) * 16) =
                    make_uint4(0, 0, 0, 0);
        }
        __syncwarp();
    }
#pragma unroll
    for (int j2 = 0; j2 < D / 32; ++j2) {
        // tokens 0 .. 7 and 8 .. 15 of sixteen dimensions, then of the next
        uint32_t b[4];
        ldsm_x4_trans(at + ((turn ^ (2 * j2)) << 4) + box_rows * D, b[0], b[1], b[2], b[3]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t y = b[2 * h], z = b[2 * h + 1];
            const uint32_t f[4] = {
                e4m3_to_f16x2(__byte_perm(y, 0u, 0x4420)), e4m3_to_f16x2(__byte_perm(y, 0u, 0x4431)),
                e4m3_to_f16x2(__byte_perm(z, 0u, 0x4420)), e4m3_to_f16x2(__byte_perm(z, 0u, 0x4431))};
#pragma unroll
            for (int r = 0; r < NR; ++r) mma_f16(st.o[2 * j2 + h][r], f, pb[r][0], pb[r][1]);
        }
    }
    if (!kAll) fence_proxy_async_smem();  // generic writes before the next TMA fill
}

// A consumer's place in its group's ring, and its waits.
struct E8Ring {
    uint8_t* slots;
    const float* scales;
    uint64_t* bars;
    int* err;
    volatile int* abort_flag;
    int slot;
    uint32_t phase;
    bool dead;  // warp-uniform: a wait ran out or the CTA aborted
    uint32_t n_pass;
    __device__ __forceinline__ void wait(uint64_t* bar, uint32_t parity, int lane) {
        if (dead) return;
        const bool ok = mbar_wait(smem_addr(bar), parity, abort_flag);
        if (__all_sync(0xffffffffu, ok)) return;
        if (lane == 0 && !*abort_flag) set_error(err, kErrTimeout);
        *abort_flag = 1;
        dead = true;
    }
};

// One item of a consumer warp, from stage s on; returns the stage that comes after.
// (Its end: see consume().)  kFills: the plan has page fills.
template <int D, int NR, bool kFills>
__device__ __forceinline__ int e8_item(const DecodeArgs& a, const ItemHead& item, int it, bool last, int s,
                                       E8Ring& rg, uint8_t* smem, uint64_t* all_bars, int warp, int lane) {
    using C = DecCfg<D, true>;
    const int gid = lane >> 2, tig = lane & 3, w4 = warp & 3, G = a.G;
    const DecodeSeg* seg = a.segs + item.seg;
    const int n_tok = seg->n_tok, rows = item.n_grp * G;
    E8State<D, NR> st;
    int lim[NR][2];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int row = r * 8 + gid;
        const bool on = row < rows;
        const float2 c = load_query_f16<D>(
            a, on ? (size_t)(r ? item.seq1 : item.seq0) * a.Hq + item.head * G + row % G : 0, on, tig, st.qb[r]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            st.c[r][e] = __shfl_sync(0xffffffffu, c.x, (2 * tig + e) * 4);
            st.up[r][e] = __shfl_sync(0xffffffffu, c.y, (2 * tig + e) * 4);
            const int j = (r * 8 + 2 * tig + e) / G;
            lim[r][e] = j < item.n_grp ? seg->grp_lim[j] : 0;
            st.m[r][e] = kNoKeys;
            st.l[r][e] = 0.f;
            st.iv[r][e] = 0x1p126f;
        }
#pragma unroll
        for (int j = 0; j < D / 16; ++j) st.o[j][r][0] = st.o[j][r][1] = st.o[j][r][2] = st.o[j][r][3] = 0.f;
    }
    // tokens that every row sees, where their pages have rows for them (rows that are
    // none see what they like)
    int all = n_tok;
    for (int j = 0; j < item.n_grp; ++j) all = min(all, seg->grp_lim[j]);
    const int box_rows = min(a.P, kStageTokens);
    int page_off = 0, n_pages = 0;
    int2 next_fills = make_int2(0, 0);  // (read a stage ahead)
    if (kFills) {
        page_off = seg->page_off;
        n_pages = seg->n_pages;
        if (s < item.s1) next_fills = e8_fills(a, page_off, n_pages, s * kStageTokens + w4 * 16);
    }
    for (; s < item.s1; s += kDecodeGroups) {
        const int slot = rg.slot, tbase = s * kStageTokens + w4 * 16;
        const bool whole = tbase + 16 <= all;
        uint32_t live = 0xffffu;
        if (kFills) {
            const int2 fills = next_fills;
            if (s + kDecodeGroups < item.s1)
                next_fills = e8_fills(a, page_off, n_pages, tbase + kDecodeGroups * kStageTokens);
            live = e8_filled(fills, a.P, tbase);
        }
        if (!whole) live &= (1u << min(max(n_tok - tbase, 0), 16)) - 1u;
        rg.wait(&rg.bars[slot], rg.phase, lane);
        if (++rg.slot == C::kStages) {
            rg.slot = 0;
            rg.phase ^= 1;
        }
        if (rg.dead) continue;
        uint8_t* tile = rg.slots + slot * C::kStageBytes;
        const float* sc = rg.scales + slot * C::kStageScales;
        uint32_t see[NR][2] = {};
        if (live == 0xffffu && whole) {
            e8_stage<D, NR, true>(st, tile, sc, live, see, box_rows, w4, lane);
        } else {
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    see[r][e] = live & ((1u << min(max(lim[r][e] - tbase, 0), 16)) - 1u);
            e8_stage<D, NR, false>(st, tile, sc, live, see, box_rows, w4, lane);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_addr(&rg.bars[C::kStages + slot]));
    }

    // the rows, eight at a time, to the closing warps
    float* red_m = reinterpret_cast<float*>(smem + C::kOffRed);
    float* red_l = red_m + kDecodeConsumerWarps * kRowsPerTile;
    float* wo = reinterpret_cast<float*>(smem + C::kOffOut) + warp * C::kPassRows * D;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int rb = r * 8;
        if (rb >= rows) break;
        // the previous pass's rows have been read
        if (rg.n_pass > 0 && !(last && rb > 0)) rg.wait(&all_bars[C::kBarOutFree], (rg.n_pass - 1) & 1, lane);
        ++rg.n_pass;
        if (rg.dead && !last) continue;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float l = st.l[r][e];
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
            const int at = 2 * tig + e;
            if (gid == 0) {
                // (without a weight either it has seen no key)
                red_m[warp * kRowsPerTile + rb + at] = st.m[r][e] == kNoKeys && l == 0.f ? -INFINITY : st.m[r][e];
                red_l[warp * kRowsPerTile + rb + at] = l * 0x1p-15f;
            }
            if (rb + at < rows) {
                // (v is 2^-126 where there is no key, else 2^-107 and more)
                const float v = power_of_two(max(-exponent_of(st.iv[r][e]) - (int)kMost, -126));
#pragma unroll
                for (int j = 0; j < D / 16; ++j)
                    *reinterpret_cast<float2*>(wo + out_pos<D>(at, j * 16 + gid * 2)) =
                        make_float2(st.o[j][r][e] * v, st.o[j][r][2 + e] * v);
            }
        }
        if (last) {
            const int sole = a.items[it].sole;
            named_bar_sync(1, C::kConsumers);
            close_rows<D, true>(a, a.items + it, seg, item.head, sole, rows, rb, smem, threadIdx.x, C::kConsumers);
            if (rb + C::kPassRows < rows) {
                named_bar_sync(1, C::kConsumers);
                continue;
            }
        }
        __syncwarp();
        if (lane == 0 && !rg.dead) mbar_arrive(smem_addr(&all_bars[C::kBarOut]));
    }
    return s;
}

template <int D, bool kFills>
__device__ void consume_e8(const DecodeArgs& a, int it0, int it1, ItemHead next, uint8_t* smem, uint64_t* all_bars,
                           volatile int* abort_flag, int warp, int lane) {
    using C = DecCfg<D, true>;
    const int gid = lane >> 2, group = warp >> 2;
    E8Ring rg = {smem + group * C::kStages * C::kStageBytes,
                 reinterpret_cast<const float*>(smem + C::kOffScales) + group * C::kStages * C::kStageScales,
                 all_bars + group * 2 * C::kStages, a.err, abort_flag, 0, 0, false, 0};
    int skip = group;  // stages to the group's next one
    for (int it = it0; it < it1; ++it) {
        const ItemHead item = next;
        if (it + 1 < it1) next.read(a, it + 1, gid / a.G, (gid + 8) / a.G);
        const bool last = it + 1 == it1;
        const int s = item.n_grp * a.G <= 8
                          ? e8_item<D, 1, kFills>(a, item, it, last, item.s0 + skip, rg, smem, all_bars, warp, lane)
                          : e8_item<D, 2, kFills>(a, item, it, last, item.s0 + skip, rg, smem, all_bars, warp, lane);
        skip = s - item.s1;
    }
}

// ---- item ends: arrivals and the merge of finished (sequence, KV head) runs ---
// Two warps close the items while the consumers stream the next ones: they add
// the consumer warps' rows (weights 2^(m_w - M), warps in order), write the
// item's partials or outputs, arrive on the runs it belongs to and merge those
// it completes.  (With the consumers doing this between items, a batch of 36
// short sequences, ~3 items per CTA, stalled at every end: 51.4 us per call
// against 46.9.)  Of a CTA's last item the consumers add and write the rows
// themselves and merge the runs it completes, since nothing is left to stream;
// the closing warps only arrive.  That shortens the chain after the last stage,
// which a call cannot hide: one sequence of 32,768 tokens 25.1 -> 24.6 us per
// call, the 36 short ones 46.9 -> 46.4.
//
// The arrival word of a run holds two counts.  Its low half counts the items
// that finished (an acquire add, the claim); the claim that brings it to the
// run's length makes its CTA the merger.  Every other CTA then publishes its
// partial with a release add to the high half, and the merger, instead of
// releasing its own partial first (a GPU-scope fence on its critical path),
// reads whether the high half counts the other entries: in the claim's own
// answer, as a rule (the last one to finish), else in acquire loads until it
// does (their claims came first, so their releases are under way: the wait
// depends on nothing this CTA still has to do); its own partial it reads back
// within the CTA.  The merger then takes all of the run's claims and releases off
// the word, also the releases still due when its own wait ran out (a store of
// zero would leave those to the next call, which could then merge too early).
// Every CTA claims once per (item, group member), also after a wait ran out, so
// every call leaves every word at zero, and a plan upload writes zeros; the word
// therefore always starts a call at zero.  A run holds at most 65,535 entries
// (the planner's limit), so the low half never carries.

// GPU-scope atomics of the arrival protocol.
__device__ __forceinline__ unsigned atom_add_acquire_gpu(unsigned* p, unsigned v) {
    unsigned old;
    asm volatile("atom.acquire.gpu.global.add.u32 %0, [%1], %2;" : "=r"(old) : "l"(p), "r"(v) : "memory");
    return old;
}
__device__ __forceinline__ void red_add_release_gpu(unsigned* p, unsigned v) {
    asm volatile("red.release.gpu.global.add.u32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
__device__ __forceinline__ unsigned ld_acquire_gpu(const unsigned* p) {
    unsigned v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

// (max, sum, weighted output) of one output float4.
struct MergeAcc {
    float M, L;
    float4 o;
    __device__ void clear() {
        M = -INFINITY;
        L = 0.f;
        o = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __device__ void rescale(float to) {  // to >= M
        const float sc = exp2f(M - (to == -INFINITY ? 0.f : to));
        L *= sc;
        o.x *= sc; o.y *= sc; o.z *= sc; o.w *= sc;
        M = to;
    }
    __device__ void add(float w, float l, const float4& v) {
        L += w * l;
        o.x += w * v.x; o.y += w * v.y; o.z += w * v.z; o.w += w * v.w;
    }
};

// One run completed by an item: its (sequence, KV head), entries [e0, e0 + n).
struct RunRef {
    int key, e0, n;
};

// A run's entries are added in two shares (the even and the odd ones), each in
// order, whoever merges it: the result does not depend on which CTA, or which
// of its warps, completes the run.  The entries come straight from L2, kBatch
// at a time.
template <int D, int kBatch>
__device__ __forceinline__ MergeAcc merge_batches(const DecodeArgs& a, const RunRef& run, int row,
                                                  int c4, int share) {
    const int G = a.G;
    const float* po = a.part_o + ((size_t)run.e0 * G + row) * D + c4 * 4;
    const float* pm = a.part_ml + ((size_t)run.e0 * G + row) * 4;
    MergeAcc acc;
    acc.clear();
    for (int e = share; e < run.n; e += 2 * kBatch) {
        float2 ml[kBatch];
        float4 o[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int x = e + 2 * u;
            if (x < run.n) {
                ml[u] = __ldcg(reinterpret_cast<const float2*>(pm + (size_t)x * G * 4));
                o[u] = __ldcg(reinterpret_cast<const float4*>(po + (size_t)x * G * D));
            } else {
                ml[u] = make_float2(-INFINITY, 0.f);
                o[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            }
        }
        float bm = acc.M;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) bm = fmaxf(bm, ml[u].x);
        acc.rescale(bm);
        const float bs = bm == -INFINITY ? 0.f : bm;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) acc.add(exp2f(ml[u].x - bs), ml[u].y, o[u]);
    }
    return acc;
}

// Long runs (one sequence spread over the GPU: ~19 entries per run) want every
// load in one round trip; short ones little besides their few entries.
template <int D>
__device__ __forceinline__ MergeAcc merge_share(const DecodeArgs& a, const RunRef& run, int row,
                                                int c4, int share) {
    return run.n <= 8 ? merge_batches<D, 4>(a, run, row, c4, share)
                      : merge_batches<D, 12>(a, run, row, c4, share);
}

// Adds the second share to the first and writes the normalised output.
template <int D>
__device__ __forceinline__ void merge_finish(const DecodeArgs& a, const RunRef& run, int row, int c4,
                                             MergeAcc x, const MergeAcc& y) {
    const float bm = fmaxf(x.M, y.M);
    x.rescale(bm);
    x.add(exp2f(y.M - (bm == -INFINITY ? 0.f : bm)), y.L, y.o);
    const int i = run.key / a.Hkv, h = (run.key % a.Hkv) * a.G + row;
    write_out(a, ((size_t)i * a.Hq + h) * D + c4 * 4, x.o, 1.f / x.L);
}

// The closing warps (et: thread 0 .. 63 of them).
template <int D, bool kE8>
__device__ void close_items(const DecodeArgs& a, int it0, int it1, uint8_t* smem, uint64_t* bars,
                            volatile int* abort_flag, int et) {
    using C = DecCfg<D, kE8>;
    constexpr int kVec = D / 4;  // float4 per output row
    const int G = a.G, lane = et & 31;
    int* n_runs = reinterpret_cast<int*>(smem + C::kOffRuns);
    RunRef* runs = reinterpret_cast<RunRef*>(n_runs + 4);
    uint32_t n_pass = 0;
    bool dead = false;  // warp-uniform
    for (int it = it0; it < it1; ++it) {
        // read while the item is streamed
        const DecodeItem* item = a.items + it;
        const DecodeSeg* seg = a.segs + item->seg;
        const int head = item->head, sole = item->sole, n_grp = seg->n_grp;
        const int rows = n_grp * G;
        // the arrival of this lane's group member (first warp)
        int key = -1;
        RunRef mine{-1, 0, 0};
        if (et < n_grp && !((sole >> et) & 1)) {
            key = seg->grp_seq[et] * a.Hkv + head;
            mine.key = key;
            mine.e0 = a.comb_off[key];
            mine.n = a.comb_off[key + 1] - mine.e0;
        }
        for (int rb = 0; rb < rows; rb += C::kPassRows, ++n_pass) {
            if (!dead) {
                const bool ok = mbar_wait(smem_addr(&bars[C::kBarOut]), n_pass & 1, abort_flag);
                if (!__all_sync(0xffffffffu, ok)) {
                    if (lane == 0 && !*abort_flag) set_error(a.err, kErrTimeout);
                    *abort_flag = 1;
                    dead = true;
                }
            }
            if (dead) continue;
            if (it + 1 == it1) break;  // the consumers have added and written its rows
            close_rows<D, kE8>(a, item, seg, head, sole, rows, rb, smem, et, C::kClosers);
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&bars[C::kBarOutFree]));
        }
        // both warps' partials are written (and the list of the item before read)
        named_bar_sync(3, C::kClosers);
        if (et < 32) {
            bool merger = false;
            if (key >= 0) {
                const unsigned old = atom_add_acquire_gpu(a.arrive + key, 1u);
                merger = (old & 0xffffu) + 1u == (unsigned)mine.n;
                if (!merger) {
                    red_add_release_gpu(a.arrive + key, kArriveRelease);
                } else if (!arrive_complete(old, mine.n)) {
                    const uint64_t t0 = globaltimer_ns();
                    for (uint32_t spin = 1;; ++spin) {
                        if (arrive_complete(ld_acquire_gpu(a.arrive + key), mine.n)) break;
                        if ((spin & 31) == 0 && globaltimer_ns() - t0 > kWaitLimitNs) {
                            set_error(a.err, kErrTimeout);
                            break;
                        }
                    }
                }
                if (merger) atomicAdd(a.arrive + key, arrive_settle(mine.n));
            }
            const unsigned mask = __ballot_sync(0xffffffffu, merger);
            if (merger) runs[__popc(mask & ((1u << lane) - 1u))] = mine;
            if (lane == 0) *n_runs = __popc(mask);
            __syncwarp();
        }
        if (it + 1 == it1) {
            if (et == 0) mbar_arrive(smem_addr(&bars[C::kBarRuns]));
            break;
        }
        named_bar_sync(3, C::kClosers);
        const int n = *reinterpret_cast<volatile int*>(n_runs);
        for (int q = 0; q < n; ++q) {
            const RunRef run = runs[q];
            for (int x = et; x < G * kVec; x += C::kClosers) {
                const int row = x / kVec, c4 = x % kVec;
                const MergeAcc s0 = merge_share<D>(a, run, row, c4, 0);
                merge_finish<D>(a, run, row, c4, s0, merge_share<D>(a, run, row, c4, 1));
            }
        }
    }
}

// The runs of the CTA's last item, by the consumers: a thread per share of an
// output, the second shares through shared memory.
template <int D, bool kE8>
__device__ void merge_last_runs(const DecodeArgs& a, uint8_t* smem, uint64_t* bars,
                                volatile int* abort_flag, int lane) {
    using C = DecCfg<D, kE8>;
    constexpr int kT = C::kConsumers, kVec = D / 4;
    const int tid = threadIdx.x;
    const int outs = a.G * kVec;  // of one run, <= 512
    const int* n_runs = reinterpret_cast<const int*>(smem + C::kOffRuns);
    volatile int* failed = const_cast<volatile int*>(n_runs + 1);
    const RunRef* runs = reinterpret_cast<const RunRef*>(n_runs + 4);
    const bool ok = mbar_wait(smem_addr(&bars[C::kBarRuns]), 0, abort_flag);
    if (!ok) {
        if (!*abort_flag) set_error(a.err, kErrTimeout);
        *abort_flag = 1;
        *failed = 1;
    }
    named_bar_sync(1, kT);  // from here on every consumer sees the same
    const int n = *failed ? 0 : *reinterpret_cast<const volatile int*>(n_runs);
    // (the item-end rows have been read: their buffer takes the shares)
    float4* x_o = reinterpret_cast<float4*>(smem + C::kOffOut);
    float2* x_ml = reinterpret_cast<float2*>(x_o + kT);
    static_assert(kT * 24 <= C::kOutBytes, "shares");
    // kT / 2 outputs at a time
    for (int b = 0; b < n * outs; b += kT / 2) {
        const int x = b + tid % (kT / 2), share = tid / (kT / 2);
        const bool on = x < n * outs;
        MergeAcc acc;
        RunRef run{};
        int row = 0, c4 = 0;
        if (on) {
            run = runs[x / outs];
            row = x % outs / kVec;
            c4 = x % kVec;
            acc = merge_share<D>(a, run, row, c4, share);
            if (share) {
                x_o[tid] = acc.o;
                x_ml[tid] = make_float2(acc.M, acc.L);
            }
        }
        named_bar_sync(1, kT);
        if (on && !share) {
            MergeAcc other;
            const float2 ml = x_ml[tid + kT / 2];
            other.M = ml.x;
            other.L = ml.y;
            other.o = x_o[tid + kT / 2];
            merge_finish<D>(a, run, row, c4, acc, other);
        }
        named_bar_sync(1, kT);
    }
}

template <int D, bool kE8>
__global__ void __launch_bounds__(DecCfg<D, kE8>::kThreads, 1)
    sq_decode_splitk_kernel(const __grid_constant__ CUtensorMap tmap,
                            const __grid_constant__ ArgsOf<kE8> a) {
    using C = DecCfg<D, kE8>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>(
        (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kOffBars);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + C::kBarRuns + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // per group: full [kStages], empty [kStages]
    if (threadIdx.x < kDecodeGroups * 2 * C::kStages) {
        // (8 bits, several pages to a stage: two arrivals for each page)
        const int filled = kE8 && a.P < kStageTokens ? 2 * kStageTokens >> (__ffs(a.P) - 1) : 1;
        mbar_init(smem_addr(&bars[threadIdx.x]),
                  threadIdx.x / C::kStages % 2 ? kDecodeConsumerWarps / kDecodeGroups : filled);
        fence_mbar_init();
    }
    if (threadIdx.x == 0) {
        mbar_init(smem_addr(&bars[C::kBarOut]), kDecodeConsumerWarps);
        mbar_init(smem_addr(&bars[C::kBarOutFree]), C::kClosers / 32);
        mbar_init(smem_addr(&bars[C::kBarRuns]), 1);
        reinterpret_cast<int*>(smem + C::kOffRuns)[1] = 0;
        *abort_flag = 0;
        fence_mbar_init();
    }
    const int group = warp - kDecodeConsumerWarps;
    if (group >= 0 && group < kDecodeGroups) {
        if (threadIdx.x == C::kConsumers) prefetch_tmap(&tmap);
        if constexpr (kE8) {
            const uint32_t slots = smem_addr(smem) + group * C::kStages * C::kStageBytes;
            const uint32_t scales = smem_addr(smem) + C::kOffScales + group * C::kStages * C::kStageScales * 4;
            const uint32_t own = smem_addr(bars + group * 2 * C::kStages);
            if (a.P >= kStageTokens) ProducerE8<D, true>{&tmap, a, slots, scales, own, abort_flag, group, lane}.live();
            else ProducerE8<D, false>{&tmap, a, slots, scales, own, abort_flag, group, lane}.live();
        } else {
            Producer<D> pr{&tmap, a, smem + group * C::kStages * C::kStageBytes,
                           bars + group * 2 * C::kStages, abort_flag, group, lane};
            // A reused plan is read before the wait.  Pages no in-flight work writes
            // (the host checked every library write to them is complete; the kernels
            // before this one write no other pool memory) are loaded before it too:
            // the first stages stream in while the previous kernel finishes.
            if (a.plan_ready) pr.init();
            named_bar_sync(2, C::kThreads);  // (the barriers are initialised)
            if (a.plan_ready) pr.early();
            grid_dependency_wait();
            grid_launch_dependents();  // the next kernel may be scheduled as CTAs retire
            if (!a.plan_ready) pr.init();
            pr.run();
        }
        return;
    }
    const bool closer = group >= kDecodeGroups;
    const int j0 = (lane >> 2) / a.G, j1 = ((lane >> 2) + 8) / a.G;
    int it0 = 0, it1 = 0;
    ItemHead head{};
    auto read_plan = [&]() {
        it0 = a.cta_begin[blockIdx.x];
        it1 = a.cta_begin[blockIdx.x + 1];
        if (it0 < it1 && !closer) head.read(a, it0, j0, j1);
    };
    if (a.plan_ready) read_plan();
    named_bar_sync(2, C::kThreads);
    // Launched as a programmatic dependent: the set-up above overlapped the
    // previous kernel's tail; nothing else it may have written is read before here.
    grid_dependency_wait();
    grid_launch_dependents();
    if (!a.plan_ready) read_plan();
    if (it0 == it1) return;
    if (closer) {
        close_items<D, kE8>(a, it0, it1, smem, bars, abort_flag,
                       threadIdx.x - C::kConsumers - kDecodeGroups * 32);
        return;
    }
    if constexpr (kE8) {
        if (a.page_fill) consume_e8<D, true>(a, it0, it1, head, smem, bars, abort_flag, warp, lane);
        else consume_e8<D, false>(a, it0, it1, head, smem, bars, abort_flag, warp, lane);
    } else consume<D>(a, it0, it1, head, smem, bars, abort_flag, warp, lane);
    merge_last_runs<D, kE8>(a, smem, bars, abort_flag, lane);
}

}  // namespace

int64_t decode_partial_bytes(int32_t n_ent, int32_t G, int32_t D) {
    return (int64_t)n_ent * G * (D + 4) * (int64_t)sizeof(float);
}

template <int D, bool kE8>
static cudaError_t prepare_one() {
    cudaError_t e = cudaFuncSetAttribute(sq_decode_splitk_kernel<D, kE8>,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize,
                                         DecCfg<D, kE8>::kSmemBytes);
    if (e != cudaSuccess) return e;
    // the largest shared-memory carveout
    return cudaFuncSetAttribute(sq_decode_splitk_kernel<D, kE8>,
                                cudaFuncAttributePreferredSharedMemoryCarveout,
                                cudaSharedmemCarveoutMaxShared);
}

cudaError_t decode_prepare(int D) {
    const cudaError_t e = D == 128 ? prepare_one<128, false>() : prepare_one<64, false>();
    if (e != cudaSuccess) return e;
    return D == 128 ? prepare_one<128, true>() : prepare_one<64, true>();
}

// (that of rows in 8 bits is the same: a CTA's shared memory leaves no room for two)
int decode_ctas_per_sm(int D) {
    int n = 0;
    cudaError_t e;
    if (D == 128)
        e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, sq_decode_splitk_kernel<128, false>,
                                                          DecCfg<128, false>::kThreads,
                                                          DecCfg<128, false>::kSmemBytes);
    else
        e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, sq_decode_splitk_kernel<64, false>,
                                                          DecCfg<64, false>::kThreads,
                                                          DecCfg<64, false>::kSmemBytes);
    if (e != cudaSuccess || n < 1) return 1;
    return n;
}

// The kernel is launched as a programmatic dependent of whatever precedes it
// on the stream: it waits (griddepcontrol.wait) before it reads anything the
// preceding work may write, so its launch and set-up overlap that work's tail.
static cudaLaunchAttribute pdl_attr() {
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    return at;
}

template <int D, bool kE8>
static cudaError_t launch_one(const CUtensorMap& tmap, const ArgsOf<kE8>& a, int n_ctas, cudaStream_t st) {
    cudaLaunchAttribute at = pdl_attr();
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(n_ctas);
    cfg.blockDim = dim3(DecCfg<D, kE8>::kThreads);
    cfg.dynamicSmemBytes = DecCfg<D, kE8>::kSmemBytes;
    cfg.stream = st;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, sq_decode_splitk_kernel<D, kE8>, tmap, a);
}

cudaError_t launch_decode(const CUtensorMap& tmap, const DecodeArgs& a, int n_ctas, int D,
                          cudaStream_t st) {
    return D == 128 ? launch_one<128, false>(tmap, a, n_ctas, st) : launch_one<64, false>(tmap, a, n_ctas, st);
}
cudaError_t launch_decode_kv8(const CUtensorMap& tmap, const DecodeKv8Args& a, int n_ctas, int D,
                              cudaStream_t st) {
    return D == 128 ? launch_one<128, true>(tmap, a, n_ctas, st) : launch_one<64, true>(tmap, a, n_ctas, st);
}

}  // namespace sq
