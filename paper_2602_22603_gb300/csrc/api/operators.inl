// The calls around a model's attention: rows added before their K/V exist, norms
// and rotation of queries and keys into the cache, attention of query blocks, and
// what stays of a drafted tree.  One translation unit with sq_api.cpp, whose cache
// object and helpers they share.  See include/sq.h for the contract of every call.

namespace {

// A call whose host side may run out of memory: what it threw as a status.
template <typename F>
int guarded(F f) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return SQ_ERR_NO_MEMORY;
    } catch (const std::length_error&) {
        return SQ_ERR_NO_MEMORY;
    }
}

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// n_seqs distinct live handles.
int check_handles(sq_cache* c, const sq_seq* seqs, int32_t n_seqs) {
    if (n_seqs < 0 || (n_seqs > 0 && !seqs)) return SQ_ERR_INVALID_ARG;
    // (a live handle's slot, its low 20 bits, is below max_seqs)
    if (c->slot_mark.empty()) c->slot_mark.assign(c->g.max_seqs, 0);
    const uint64_t mark = ++c->mark;
    for (int32_t i = 0; i < n_seqs; ++i)
        if (!c->host->seq(seqs[i])) return SQ_ERR_BAD_HANDLE;
    for (int32_t i = 0; i < n_seqs; ++i) {
        uint64_t& m = c->slot_mark[seqs[i] & 0xfffff];
        if (m == mark) return SQ_ERR_INVALID_ARG;
        m = mark;
    }
    return SQ_OK;
}

// The newest rows of each sequence that a call is about (counts NULL: one each):
// between 0 and the sequence's rows.  *total = their number.
int check_counts(sq_cache* c, const sq_seq* seqs, int32_t n_seqs, const int32_t* counts, int64_t* total) {
    *total = 0;
    for (int32_t i = 0; i < n_seqs; ++i) {
        const int32_t m = counts ? counts[i] : 1;
        if (m < 0 || m > c->host->seq(seqs[i])->n) return SQ_ERR_INVALID_ARG;
        *total += m;
    }
    return *total > 0x7fffffff ? SQ_ERR_INVALID_ARG : SQ_OK;
}

// The bytes of n rows of row_elems bf16 each, stride elements apart.
size_t rows_bytes(int64_t n, int64_t row_elems, int64_t stride) {
    return n > 0 ? (size_t)((n - 1) * stride + row_elems) * 2 : 0;
}

struct Range {
    const void* p;
    size_t n;
};
// True when an output overlaps an input or another output.
bool any_overlap(const std::vector<Range>& in, const std::vector<Range>& out) {
    for (size_t i = 0; i < out.size(); ++i) {
        for (const Range& r : in)
            if (overlaps(out[i].p, out[i].n, r.p, r.n)) return true;
        for (size_t j = 0; j < i; ++j)
            if (overlaps(out[i].p, out[i].n, out[j].p, out[j].n)) return true;
    }
    return false;
}

// True when rows of aw and of bw elements, equally far apart, take turns (parts of
// one fused tensor).
bool rows_take_turns(const void* a, int64_t aw, int64_t as, const void* b, int64_t bw, int64_t bs) {
    const int64_t d = (int64_t)(reinterpret_cast<intptr_t>(b) - reinterpret_cast<intptr_t>(a)) / 2;
    return as == bs && ((d >= aw && d + bw <= as) || (-d >= bw && aw - d <= as));
}

bool rows_ok(const void* p, int64_t stride, int64_t row_elems) {
    return p && aligned(p, 16) && stride >= row_elems && stride % 8 == 0 && stride < (int64_t(1) << 40);
}

int check_params(const Geometry& g, const sq_norm_rope* p, const int32_t* positions, bool need_positions) {
    if (!p || !aligned(p->q_weight, 16) || !aligned(p->k_weight, 16) || !aligned(positions, 4))
        return SQ_ERR_INVALID_ARG;
    if (p->weight_dtype != SQ_OUT_BF16 && p->weight_dtype != SQ_OUT_F32) return SQ_ERR_INVALID_ARG;
    if (p->rot_dim < 0 || p->rot_dim > g.D || p->rot_dim % 16 != 0) return SQ_ERR_INVALID_ARG;
    if (!(p->eps >= 0.f) || p->eps > 3.0e38f) return SQ_ERR_INVALID_ARG;
    if (p->rot_dim > 0) {
        if (!p->rope || !aligned(p->rope, 16) || p->max_pos < 1) return SQ_ERR_INVALID_ARG;
        if (need_positions && !positions) return SQ_ERR_INVALID_ARG;
    }
    return SQ_OK;
}

template <typename Args>
void fill_params(sq_cache* c, const sq_norm_rope* p, Args* a) {
    a->q_weight = p->q_weight;
    a->k_weight = p->k_weight;
    a->weight_f32 = p->weight_dtype == SQ_OUT_F32;
    a->rope = reinterpret_cast<const float2*>(p->rope);
    a->rot = p->rot_dim;
    a->interleaved = p->interleaved ? 1 : 0;
    a->max_pos = p->max_pos;
    a->eps = p->eps;
    a->Hq = c->g.Hq;
    a->Hkv = c->g.Hkv;
    a->err = c->d_err;
}

const __nv_bfloat16* bf16(const void* p) { return reinterpret_cast<const __nv_bfloat16*>(p); }
__nv_bfloat16* bf16(void* p) { return reinterpret_cast<__nv_bfloat16*>(p); }

// A buffer of the cache that calls on any stream take turns with: `bytes` of it,
// usable by work on `st` from here on.  While `st` is captured: what there is, for
// the graph to keep.
int take_buffer(sq_cache* c, TurnBuffer& b, size_t bytes, cudaStream_t st, bool captured) {
    cudaError_t e;
    if (captured) {
        if (bytes > b.cap) return SQ_ERR_UNSUPPORTED;
        b.captured = true;
        return SQ_OK;
    }
    if (!b.ev) {
        e = cudaEventCreateWithFlags(&b.ev, cudaEventDisableTiming);
        if (e != cudaSuccess) return cuda_status(e);
    }
    if (bytes > b.cap) {
        if (b.ev_recorded) cudaEventSynchronize(b.ev);
        retire(c, b.d, b.captured);
        b.d = nullptr;
        b.cap = 0;
        b.ev_recorded = b.captured = false;
        const size_t cap = std::max<size_t>(bytes * 5 / 4, 4096);
        e = cudaMalloc(&b.d, cap);
        if (e != cudaSuccess) {
            cudaGetLastError();
            return cuda_status(e);
        }
        b.cap = cap;
    }
    if (b.ev_recorded && b.ev_stream != st) {
        e = cudaStreamWaitEvent(st, b.ev, 0);
        if (e != cudaSuccess) return cuda_status(e);
    }
    return SQ_OK;
}

// After the work that uses it has been enqueued (or may have been).
int used_buffer(TurnBuffer& b, cudaStream_t st, bool captured) {
    if (captured) return SQ_OK;
    const cudaError_t e = cudaEventRecord(b.ev, st);
    if (e != cudaSuccess) {
        cudaStreamSynchronize(st);
        cudaGetLastError();
        b.ev_recorded = false;
        return cuda_status(e);
    }
    b.ev_recorded = true;
    b.ev_stream = st;
    return SQ_OK;
}

// Stamps pages that a store writes.  Their sequences keep their versions, so
// plans made before do not list these writes: the cache does (early_writes), the
// pages of the newest store one by one.
void note_store(sq_cache* c, std::vector<int32_t>&& pages, void* stream) {
    if (!c->early_ok) return;
    const bool again = pages == c->store_pages;
    if (again && stream == c->store_stream && !c->write_pending.empty() &&
        c->write_pending.back().first == c->store_ticket && !capturing(as_stream(stream))) {
        // The store before was the last write, to the same pages (the next layer's): its
        // event moves on, since nothing may read them ahead of this one either.  (With
        // events of its own for every store, looked after 32 at a time, one of a single
        // token took 10.5 us instead of 8.8.)
        const uint64_t t = ++c->write_seq;
        if (cudaEventRecord(c->write_pending.back().second, as_stream(stream)) != cudaSuccess) {
            cudaGetLastError();
            c->early_ok = false;
            return;
        }
        for (int32_t p : pages) c->page_ticket[p] = t;
        c->write_pending.back().first = c->store_ticket = t;
        return;
    }
    // (stores may go on without an attention call, which would look after them)
    if (c->write_pending.size() >= 32 && !capturing(as_stream(stream))) poll_writes(c);
    note_writes(c, pages.data(), pages.size(), stream);
    c->store_stream = stream;
    if (!again) {
        c->store_rest = c->store_ticket;
        c->store_pages = std::move(pages);
    }
    c->store_ticket = c->write_seq;
}

// `rows`, where there is one, is enqueued after the copies, with the rows counted, and
// notes its writes; where it fails they are taken back.
template <typename Rows>
int extend_impl(sq_cache* c, const sq_seq* seqs, int32_t n_seqs, const int32_t* n_new, void* stream, Rows rows) {
    constexpr bool kLater = std::is_same<Rows, std::nullptr_t>::value;  // (their rows come later)
    int rc = check_handles(c, seqs, n_seqs);
    if (rc != SQ_OK) return rc;
    int64_t total = 0;
    for (int32_t i = 0; i < n_seqs; ++i) {
        if (n_new && n_new[i] < 0) return SQ_ERR_INVALID_ARG;
        total += n_new ? n_new[i] : 1;
    }
    if (total == 0) return SQ_OK;
    const Geometry& g = c->g;
    cudaStream_t st = as_stream(stream);
    std::vector<AppendPlan> plans(n_seqs);
    std::vector<uint64_t> old_versions(n_seqs);
    std::vector<std::vector<LenUpdate>> ups(n_seqs);
    std::vector<char> passed(n_seqs, 0);
    std::vector<int32_t> taken, copied, left;
    std::vector<CowCopy> copies;
    // takes back what was planned, unless everything is enqueued.  What is under way then
    // (copies into pages that are free again, words of plans that other calls may
    // replace) is waited for; in a captured call it does not run.
    struct Undo {
        HostCache* host;
        const sq_seq* seqs;
        const std::vector<AppendPlan>* plans;
        int32_t planned;
        bool enqueued;
        cudaStream_t st;
        ~Undo() {
            if (planned > 0 && enqueued && !capturing(st)) {
                cudaStreamSynchronize(st);
                cudaGetLastError();
            }
            for (int32_t j = planned - 1; j >= 0; --j) host->undo_append(seqs[j], (*plans)[j]);
        }
    } undo = {c->host.get(), seqs, &plans, 0, false, st};
    for (int32_t i = 0; i < n_seqs; ++i) {
        old_versions[i] = c->host->seq(seqs[i])->version;
        rc = c->host->append(seqs[i], n_new ? n_new[i] : 1, &plans[i]);
        if (rc != SQ_OK) return rc;
        undo.planned = i + 1;
        const AppendPlan& p = plans[i];
        taken.insert(taken.end(), p.taken.begin(), p.taken.end());
        if (p.cow) {
            copies.push_back({p.cow_old, p.cow_new, p.cow_rows});
            copied.push_back(p.cow_new);
            if (c->kv8) left.push_back(p.cow_old);
        } else if (c->kv8 && p.last_fill0 > 0 && !p.pages.empty()) {
            taken.push_back(p.pages[0]);   // (its rows may change their scale)
        }
    }
    // cached decode plans that the longer sequences leave valid: their row limits
    // go with the launch, as an append's do
    for (int32_t i = 0; i < n_seqs; ++i)
        if (plans[i].n_new > 0) plan_len_updates(c, seqs[i], plans[i], old_versions[i], st, &ups[i]);
    rc = fence_taken_pages(c, taken, stream);
    if (rc != SQ_OK) return rc;
    AppendBatchArgs a;
    a.pool = c->pool;
    a.k = a.v = nullptr;
    a.num_pages = g.num_pages;
    a.L = g.L; a.Hkv = g.Hkv; a.P = g.P; a.D = g.D;
    a.n_total = a.row0 = a.n = 0;
    a.err = c->d_err;
    a.lens.n = 0;
    for (int32_t i = 0; i < n_seqs; ++i) {
        AppendLens part;
        int words = 0;
        for (const LenUpdate& u : ups[i]) words += update_words(u);
        if (words == 0 || a.lens.n + words > kAppendLenMax) continue;
        fill_lens(ups[i], 0, &part);
        for (int32_t k = 0; k < part.n; ++k) {
            a.lens.ptr[a.lens.n] = part.ptr[k];
            a.lens.val[a.lens.n++] = part.val[k];
        }
        passed[i] = 1;
    }
    for (size_t b = 0; b < copies.size() || a.lens.n > 0; b += kAppendBatchMax) {
        a.n_cow = b < copies.size() ? (int32_t)std::min<size_t>(kAppendBatchMax, copies.size() - b) : 0;
        std::copy_n(copies.begin() + std::min(b, copies.size()), a.n_cow, a.cow);
        cudaError_t e;
        if (c->kv8) {
            Kv8CopyArgs ca;
            ca.pool = kv8_pool(c);
            ca.L = g.L;
            ca.lens = a.lens;
            ca.n_cow = a.n_cow;
            std::copy_n(a.cow, a.n_cow, ca.cow);
            ca.err = c->d_err;
            e = launch_kv8_copy(ca, g.D, st);
        } else {
            e = launch_append_batch(a, st);
        }
        if (e != cudaSuccess) return cuda_status(e);
        undo.enqueued = true;
        a.lens.n = 0;
    }
    if constexpr (!kLater) {
        rc = rows();
        if (rc != SQ_OK) return rc;
    }
    undo.planned = 0;
    note_writes(c, copied.data(), copied.size(), stream);
    rc = record_freed(c, left, stream);
    for (int32_t i = 0; i < n_seqs; ++i) {
        if (plans[i].n_new == 0) continue;
        if (kLater) c->host->seq_mut(seqs[i])->extended = true;
        const uint64_t nv = c->host->seq(seqs[i])->version;
        if (passed[i])
            for (const LenUpdate& u : ups[i]) plan_len_apply(c, u, nv, plans[i].n_new, plans[i].pages[0], st);
        c->host->seq_mut(seqs[i])->last_stream = stream;
        if (plans[i].cow) c->stats.cow_pages += 1;
    }
    c->stats.appended_tokens += total;
    return rc;
}

// Where the newest n_new[i] rows of each sequence lie, sequence after sequence,
// and their pages (`places` may be null).
void list_places(sq_cache* c, const sq_seq* seqs, int32_t n_seqs, const int32_t* n_new, int64_t n,
                 std::vector<RowPlace>* places, std::vector<int32_t>* pages) {
    const int32_t P = c->g.P;
    if (places) places->resize((size_t)n);
    RowPlace* out = places ? places->data() : nullptr;
    for (int32_t i = 0; i < n_seqs; ++i) {
        const Seq* s = c->host->seq(seqs[i]);
        int32_t m = n_new ? n_new[i] : 1;
        int64_t pos = s->next_pos;
        if (out) out += m;
        RowPlace* end = out;
        for (size_t p = s->pages.size(); m > 0; --p) {
            const int32_t page = s->pages[p - 1], k = std::min(m, s->fill[p - 1]);
            pages->push_back(page);
            m -= k;
            if (!out) continue;
            const int32_t row = page * P + s->fill[p - 1];
            for (int32_t x = 1; x <= k; ++x) *--end = {row - x, (int32_t)std::min<int64_t>(--pos, 0x7fffffff)};
        }
    }
}

// The newest n_new[i] rows of each sequence as runs, and their pages.
void list_runs(sq_cache* c, const sq_seq* seqs, int32_t n_seqs, const int32_t* n_new, std::vector<RowRun>* runs,
               std::vector<int32_t>* pages) {
    const int32_t P = c->g.P, most = std::min(P, kRunRows);
    int32_t first = 0;
    for (int32_t i = 0; i < n_seqs; ++i) {
        const Seq* s = c->host->seq(seqs[i]);
        const int32_t m = n_new ? n_new[i] : 1;
        int32_t left = m;
        for (size_t p = s->pages.size(); left > 0; --p) {
            int32_t end = s->fill[p - 1];
            const int32_t low = std::max(0, end - left);
            if (pages) pages->push_back(s->pages[p - 1]);
            while (runs && end > low) {
                const int32_t from = std::max(low, (end - 1) & ~(most - 1));
                const int32_t at = left - (s->fill[p - 1] - from);  // of the sequence's, counted from its first
                runs->push_back({s->pages[p - 1] * P + from, first + at, end - from,
                                 (int32_t)std::min<int64_t>(s->next_pos - m + at, 0x7fffffff)});
                end = from;
            }
            left -= std::min(left, s->fill[p - 1]);
        }
        first += m;
    }
}

// What a store's launch is told of its runs.
void set_runs(const std::vector<RowRun>& runs, Kv8StoreArgs* a) {
    a->n_runs = (int32_t)runs.size();
    a->blocks = a->most = 0;
    for (const RowRun& r : runs) {
        const int32_t s0 = r.row % kScaleRows, blocks = (s0 + r.n + kScaleRows - 1) / kScaleRows;
        a->blocks = std::max(a->blocks, blocks);
        a->most = std::max(a->most, blocks > 2 ? kScaleRows : blocks == 1 ? r.n : std::max(kScaleRows - s0, s0 + r.n - kScaleRows));
    }
}

int store_impl(sq_cache* c, const sq_seq* seqs, int32_t n_seqs, const int32_t* n_new, int32_t layer,
               const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
               int64_t v_stride, const int32_t* positions, const sq_norm_rope* params, void* q_out,
               void* stream) {
    if (!(c->kv8 ? (void*)launch_kv8_store : (void*)launch_norm_rope)) return SQ_ERR_UNSUPPORTED;
    const Geometry& g = c->g;
    int64_t n = 0;
    int rc = check_handles(c, seqs, n_seqs);
    if (rc == SQ_OK) rc = check_counts(c, seqs, n_seqs, n_new, &n);
    if (rc == SQ_OK) rc = check_params(g, params, positions, false);
    if (rc != SQ_OK) return rc;
    if (layer < 0 || layer >= g.L) return SQ_ERR_INVALID_ARG;
    if (n == 0) return SQ_OK;
    const int64_t qw = (int64_t)g.Hq * g.D, kw = (int64_t)g.Hkv * g.D;
    if (!rows_ok(q, q_stride, qw) || !rows_ok(k, k_stride, kw) || !rows_ok(v, v_stride, kw) ||
        !rows_ok(q_out, qw, qw))
        return SQ_ERR_INVALID_ARG;
    if (any_overlap({{q, rows_bytes(n, qw, q_stride)}, {k, rows_bytes(n, kw, k_stride)},
                     {v, rows_bytes(n, kw, v_stride)}},
                    {{q_out, rows_bytes(n, qw, qw)}, {c->pool, c->pool_bytes}}))
        return SQ_ERR_INVALID_ARG;
    // where each row goes (8-bit caches: each block's rows); more places than go with
    // the launch stay on the device for the next layer's store
    std::vector<RowPlace> places;
    std::vector<RowRun> runs;
    std::vector<int32_t> pages;
    if (c->kv8) list_runs(c, seqs, n_seqs, n_new, &runs, &pages);
    const bool upload_places = c->kv8 ? runs.size() > (size_t)kRunsInline : n > kNormInline;
    const bool captured = upload_places && capturing(as_stream(stream));
    StorePlanEntry* hit = nullptr;
    for (auto& p : c->store_plans) {
        if (!upload_places || !p.valid || (int32_t)p.handles.size() != n_seqs) continue;
        bool same = true;
        for (int32_t i = 0; i < n_seqs && same; ++i)
            same = p.handles[i] == seqs[i] && p.versions[i] == c->host->seq(seqs[i])->version &&
                   p.counts[i] == (n_new ? n_new[i] : 1);
        if (same) hit = &p;
    }
    if (!c->kv8) list_places(c, seqs, n_seqs, n_new, n, hit ? nullptr : &places, &pages);
    for (int32_t p : pages)
        if (c->host->alloc().refcount(p) > 1) return SQ_ERR_INVALID_ARG;
    cudaStream_t st = as_stream(stream);
    if (c->kv8) {
        // (see record_freed; runs of a graph take turns by the caller's order)
        bool marked = false;
        for (int32_t p : pages) marked |= c->fenced[p] != 0;
        if (marked && !capturing(st)) rc = fence_taken_pages(c, pages, stream);
        if (rc != SQ_OK) return rc;
    }
    auto launch = [&](const uint8_t* uploaded) {
        if (c->kv8) {
            Kv8StoreInlineArgs a;
            a.q = bf16(q);
            a.k = bf16(k);
            a.v = bf16(v);
            a.q_stride = q_stride;
            a.k_stride = k_stride;
            a.v_stride = v_stride;
            a.layer_stride = 0;
            a.positions = positions;
            a.runs = reinterpret_cast<const RowRun*>(uploaded);
            a.q_out = bf16(q_out);
            a.pool = kv8_pool(c);
            set_runs(runs, &a);
            a.layer = layer;
            a.n_layers = 1;
            a.plain = 0;
            fill_params(c, params, &a);
            if (!uploaded) std::copy(runs.begin(), runs.end(), a.inline_run);
            return launch_kv8_store(a, g.D, st);
        }
        NormRopeInlineArgs a;
        a.q = bf16(q);
        a.k = bf16(k);
        a.v = bf16(v);
        a.q_stride = q_stride;
        a.k_stride = k_stride;
        a.v_stride = v_stride;
        a.positions = positions;
        a.places = reinterpret_cast<const RowPlace*>(uploaded);
        a.q_out = bf16(q_out);
        a.k_out = nullptr;
        a.pool = c->pool;
        a.num_pages = g.num_pages;
        a.n = (int32_t)n;
        a.P = g.P;
        a.layer = layer;
        fill_params(c, params, &a);
        if (uploaded) return launch_norm_rope(a, g.D, true, st);
        std::copy(places.begin(), places.end(), a.inline_place);
        return launch_norm_rope_inline(a, g.D, st);
    };
    cudaError_t e;
    if (!upload_places) {
        e = launch(nullptr);
        if (e != cudaSuccess) return cuda_status(e);
    } else {
        const bool fresh = !hit;
        // (a graph takes places that are there, uploaded on its stream)
        if (captured && (fresh || hit->buf.ev_stream != st)) return SQ_ERR_UNSUPPORTED;
        if (captured) keep_captured(c->store_plans, *hit);
        if (fresh) {
            hit = entry_to_replace(c->store_plans);
            hit->valid = false;
        }
        const size_t bytes = c->kv8 ? runs.size() * sizeof(RowRun) : (size_t)n * sizeof(RowPlace);
        rc = take_buffer(c, hit->buf, bytes, st, captured);
        if (rc != SQ_OK) return rc;
        if (fresh)
            rc = staged_copy(c, hit->buf.d, c->kv8 ? (const void*)runs.data() : places.data(), bytes, stream);
        e = cudaSuccess;
        if (rc == SQ_OK) e = launch(hit->buf.d);
        const int used = used_buffer(hit->buf, st, captured);
        if (rc != SQ_OK || e != cudaSuccess || used != SQ_OK) {
            hit->valid = false;
            return rc != SQ_OK ? rc : (e != cudaSuccess ? cuda_status(e) : used);
        }
        if (fresh) {
            hit->handles.assign(seqs, seqs + n_seqs);
            hit->versions.resize(n_seqs);
            hit->counts.resize(n_seqs);
            for (int32_t i = 0; i < n_seqs; ++i) {
                hit->versions[i] = c->host->seq(seqs[i])->version;
                hit->counts[i] = n_new ? n_new[i] : 1;
            }
            hit->valid = true;
        }
        hit->last_use = ++c->use_clock;
    }
    note_store(c, std::move(pages), stream);
    for (int32_t i = 0; i < n_seqs; ++i) c->host->seq_mut(seqs[i])->last_stream = stream;
    return SQ_OK;
}

int norm_impl(sq_cache* c, int32_t n_tokens, const void* q, int64_t q_stride, const void* k,
              int64_t k_stride, const int32_t* positions, const sq_norm_rope* params, void* q_out,
              void* k_out, void* stream) {
    if (!launch_norm_rope) return SQ_ERR_UNSUPPORTED;
    const Geometry& g = c->g;
    if (n_tokens < 0) return SQ_ERR_INVALID_ARG;
    int rc = check_params(g, params, positions, n_tokens > 0);
    if (rc != SQ_OK) return rc;
    if (n_tokens == 0) return SQ_OK;
    const int64_t qw = (int64_t)g.Hq * g.D, kw = (int64_t)g.Hkv * g.D, n = n_tokens;
    if (!rows_ok(q, q_stride, qw) || !rows_ok(k, k_stride, kw) || !rows_ok(q_out, qw, qw) ||
        !rows_ok(k_out, kw, kw))
        return SQ_ERR_INVALID_ARG;
    if (any_overlap({{q, rows_bytes(n, qw, q_stride)}, {k, rows_bytes(n, kw, k_stride)}},
                    {{q_out, rows_bytes(n, qw, qw)}, {k_out, rows_bytes(n, kw, kw)}}))
        return SQ_ERR_INVALID_ARG;
    NormRopeArgs a = {};
    a.q = bf16(q);
    a.k = bf16(k);
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.positions = positions;
    a.q_out = bf16(q_out);
    a.k_out = bf16(k_out);
    a.n = n_tokens;
    fill_params(c, params, &a);
    return cuda_status(launch_norm_rope(a, g.D, false, as_stream(stream)));
}

int norm_backward_impl(sq_cache* c, int32_t n_tokens, const void* q, int64_t q_stride, const void* k,
                       int64_t k_stride, const int32_t* positions, const sq_norm_rope* params,
                       const void* dq_out, const void* dk_out, void* dq, int64_t dq_stride, void* dk,
                       int64_t dk_stride, float* dq_weight, float* dk_weight, void* stream) {
    if (!launch_norm_rope_grad) return SQ_ERR_UNSUPPORTED;
    const Geometry& g = c->g;
    if (n_tokens < 0 || !aligned(dq_weight, 4) || !aligned(dk_weight, 4)) return SQ_ERR_INVALID_ARG;
    int rc = check_params(g, params, positions, n_tokens > 0);
    if (rc != SQ_OK) return rc;
    const bool weights = dq_weight || dk_weight;
    if (n_tokens == 0 && !weights) return SQ_OK;
    const int64_t qw = (int64_t)g.Hq * g.D, kw = (int64_t)g.Hkv * g.D, n = n_tokens;
    if (n > 0 && (!rows_ok(q, q_stride, qw) || !rows_ok(k, k_stride, kw) || !rows_ok(dq_out, qw, qw) ||
                  !rows_ok(dk_out, kw, kw) || !rows_ok(dq, dq_stride, qw) || !rows_ok(dk, dk_stride, kw)))
        return SQ_ERR_INVALID_ARG;
    {
        std::vector<Range> in = {{q, rows_bytes(n, qw, q_stride)}, {k, rows_bytes(n, kw, k_stride)},
                                 {dq_out, rows_bytes(n, qw, qw)}, {dk_out, rows_bytes(n, kw, kw)}};
        std::vector<Range> out;
        const size_t wb = (size_t)g.D * 4;
        if (dq_weight) out.push_back({dq_weight, wb});
        if (dk_weight) out.push_back({dk_weight, wb});
        if (any_overlap(in, out)) return SQ_ERR_INVALID_ARG;
        // (dq and dk may be parts of one fused gradient, a row of each in turn)
        const Range rq = {dq, rows_bytes(n, qw, dq_stride)}, rk = {dk, rows_bytes(n, kw, dk_stride)};
        in.insert(in.end(), out.begin(), out.end());
        if (any_overlap(in, {rq}) || any_overlap(in, {rk})) return SQ_ERR_INVALID_ARG;
        if (overlaps(rq.p, rq.n, rk.p, rk.n) && !rows_take_turns(dq, qw, dq_stride, dk, kw, dk_stride))
            return SQ_ERR_INVALID_ARG;
    }
    cudaStream_t st = as_stream(stream);
    NormRopeGradArgs a = {};
    a.q = bf16(q);
    a.k = bf16(k);
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.positions = positions;
    a.dq_out = bf16(dq_out);
    a.dk_out = bf16(dk_out);
    a.dq = bf16(dq);
    a.dk = bf16(dk);
    a.dq_stride = dq_stride;
    a.dk_stride = dk_stride;
    a.dq_weight = dq_weight;
    a.dk_weight = dk_weight;
    a.n = n_tokens;
    a.ctas = norm_rope_grad_ctas(n_tokens, g.Hq, g.Hkv, g.D, c->num_sms);
    fill_params(c, params, &a);
    if (!weights) return cuda_status(launch_norm_rope_grad(a, g.D, st));
    const bool captured = capturing(st);
    rc = take_buffer(c, c->norm_part, (size_t)a.ctas * 2 * g.D * sizeof(float), st, captured);
    if (rc != SQ_OK) return rc;
    a.part = reinterpret_cast<float*>(c->norm_part.d);
    const cudaError_t e = launch_norm_rope_grad(a, g.D, st);
    rc = used_buffer(c->norm_part, st, captured);
    return e != cudaSuccess ? cuda_status(e) : rc;
}

// (8-bit caches) Query tiles of a sequence up to which each is a block of its own, whose
// keys and values the kernel converts: up to three the conversions cost less than the
// pages widened in memory, though every tile has its own.  32/8 heads of 128 dimensions,
// two, three and four tiles over 60,000 tokens: 86, 122 and 156 us against 117, 161 and
// 154; over 8,000 25, 31 and 36 against 24, 31 and 29; 8 sequences of 1 .. 96 queries over
// 8,000 71 against 128.  64/8 heads of 64 over 60,000: 73, 104 and 135 against 83, 144 and
// 123; over 8,000 22, 29 and 33 against 20, 26 and 26.  (The rule takes no account of the
// context: at 8,000 tokens two tiles, and of 64 dimensions two and three, lose 1 to 3 us.)
constexpr int32_t kWideTiles = 3;

// The pages of a plan as bf16, in the order of its list, as a pool of one layer.  Blocks
// of two query tiles are the tensor cores' bound, and every page serves many of them:
// it is widened once, before them (with the kernel's own converters, as one-tile blocks
// have them, 512 queries over 60,001 tokens, 32/8 heads of 128, take 555 us against 420,
// a prompt of 8,191 525 against 373).
int widen_pages(sq_cache* c, const BlockPlanEntry& plan, int32_t layer, cudaStream_t st, bool captured,
                CUtensorMap* map) {
    const Geometry& g = c->g;
    const size_t page = (size_t)2 * g.Hkv * g.P * g.D * sizeof(__nv_bfloat16);
    int rc = take_buffer(c, c->wide, plan.n_wide * page, st, captured);
    if (rc != SQ_OK) return rc;
    rc = make_pool_map(c, c->wide.d, 2, 64, plan.n_wide, 1, map);
    if (rc != SQ_OK) return rc;
    Kv8WidenArgs a;
    a.pool = kv8_pool(c);
    a.pages = reinterpret_cast<const int32_t*>(plan.d + plan.o_wide);
    a.n = plan.n_wide;
    a.layer = layer;
    a.out = bf16(static_cast<void*>(c->wide.d));
    a.err = c->d_err;
    return cuda_status(launch_kv8_widen(a, g.D, st));
}

// Attention of query blocks; parents null: sliding windows alone.
int blocks_impl(sq_cache* c, const sq_seq* seqs, int32_t n_seqs, const int32_t* n_q, const int32_t* parents,
                int32_t layer, const void* q, void* out, int32_t out_dtype, float* lse, float sm_scale,
                int32_t window, int32_t n_sink, void* stream) {
    if (!launch_blocks) return SQ_ERR_UNSUPPORTED;
    const Geometry& g = c->g;
    int64_t n = 0;
    int rc = check_handles(c, seqs, n_seqs);
    if (rc == SQ_OK) rc = check_counts(c, seqs, n_seqs, n_q, &n);
    if (rc != SQ_OK) return rc;
    if (layer < 0 || layer >= g.L || window < 0 || n_sink < 0) return SQ_ERR_INVALID_ARG;
    if (out_dtype != SQ_OUT_BF16 && out_dtype != SQ_OUT_F32) return SQ_ERR_INVALID_ARG;
    if (!(sm_scale >= 0.f) || sm_scale > 3.0e38f) return SQ_ERR_INVALID_ARG;
    if (n == 0) return SQ_OK;
    if (!q || !out || !aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4)) return SQ_ERR_INVALID_ARG;
    const size_t rows = (size_t)n * g.Hq;
    if (any_overlap({{q, rows * g.D * 2}}, {{out, rows * g.D * (out_dtype == SQ_OUT_F32 ? 4 : 2)},
                                            {lse, lse ? rows * 4 : 0}}))
        return SQ_ERR_INVALID_ARG;
    // Single tokens take the decode kernel, which wastes nothing on the 128 rows of
    // a query tile and merges in its own launch (it leaves no log-sum-exps): 48
    // tokens at windows of 4,096 rows, 8 x 128: 108 -> 72 us; one at 128: 7.6 -> 6.7.
    if (!parents && !lse && n <= n_seqs && std::all_of(n_q, n_q + (n_q ? n_seqs : 0), [](int32_t m) { return m < 2; })) {
        std::vector<sq_seq> one(seqs, seqs + n_seqs);
        if (n_q) {
            size_t k = 0;
            for (int32_t i = 0; i < n_seqs; ++i)
                if (n_q[i]) one[k++] = seqs[i];
            one.resize(k);
        }
        return decode_impl(c, one.data(), (int32_t)one.size(), layer, q, out, out_dtype, sm_scale, window,
                           n_sink, stream);
    }
    // the call as a plan knows it
    std::vector<int32_t> key;
    key.reserve(2 + 2 * n_seqs + (parents ? n : 0));
    key.push_back(window);
    key.push_back(n_sink);
    for (int32_t i = 0; i < n_seqs; ++i) key.push_back(n_q ? n_q[i] : 1);
    if (parents) {
        for (int32_t i = 0, at = 0; i < n_seqs; at += n_q[i++]) {
            if (n_q[i] > SQ_MAX_DRAFT) return SQ_ERR_INVALID_ARG;
            for (int32_t j = 0; j < n_q[i]; ++j)
                if (parents[at + j] < -1 || parents[at + j] >= j) return SQ_ERR_INVALID_ARG;
        }
        key.insert(key.end(), parents, parents + n);
    }
    cudaStream_t st = as_stream(stream);
    cudaError_t e;
    BlockPlanEntry* hit = nullptr;
    for (auto& p : c->block_plans) {
        if (!p.valid || (int32_t)p.handles.size() != n_seqs || p.tree != (parents != nullptr) ||
            p.call != key)
            continue;
        bool same = true;
        for (int32_t i = 0; i < n_seqs && same; ++i)
            same = p.handles[i] == seqs[i] && p.versions[i] == c->host->seq(seqs[i])->version;
        if (same) {
            hit = &p;
            break;
        }
    }
    int32_t plan_ready = 0;
    // (a graph takes a kept plan of its own stream, or none)
    const bool captured = capturing(st);
    if (captured && (!hit || (hit->ev_recorded && hit->ev_stream != st))) return SQ_ERR_UNSUPPORTED;
    if (!hit) {
        std::vector<BlockSeq> in(n_seqs);
        for (int32_t i = 0, at = 0; i < n_seqs; ++i) {
            in[i] = {c->host->seq(seqs[i]), n_q ? n_q[i] : 1, parents ? parents + at : nullptr};
            at += in[i].n_q;
        }
        BlockPlanHost plan;
        const int32_t most_one = c->kv8 ? kWideTiles : 1;
        rc = plan_blocks(g, in, window, n_sink, c->num_sms, kPrefillPartLimit, &plan, most_one);
        if (rc == SQ_OK && plan.n_parts > 0) {
            rc = reserve_parts(c, (size_t)plan.n_parts * prefill_part_bytes(g.D));
            // no room for partial results: the plan without any
            if (rc == SQ_ERR_NO_MEMORY)
                rc = plan_blocks(g, in, window, n_sink, c->num_sms, 0, &plan, most_one);
        }
        if (rc != SQ_OK) return rc;
        std::vector<int32_t> read, wide;
        for (int32_t p : plan.tile_pages)
            if (p >= 0 && (read.empty() || read.back() != p)) read.push_back(p);
        // (8-bit caches, blocks of two tiles) the pages are widened for the call; its
        // tiles name them by their places in the list
        if (c->kv8 && !plan.one) {
            std::unordered_map<int32_t, int32_t> place;
            for (int32_t& p : plan.tile_pages) {
                if (p < 0) continue;
                const auto at = place.emplace(p, (int32_t)wide.size());
                if (at.second) wide.push_back(p);
                p = at.first->second;
            }
        }
        // upload: the records of 16 bytes first, so that each part is aligned
        struct Part {
            const void* p;
            size_t bytes, at;
        } parts[] = {{plan.tiles.data(), plan.tiles.size() * sizeof(PrefillTile), 0},
                     {plan.items.data(), plan.items.size() * sizeof(BlockItem), 0},
                     {plan.merges.data(), plan.merges.size() * sizeof(BlockMerge), 0},
                     {plan.rows.data(), plan.rows.size() * sizeof(int32_t), 0},
                     {plan.bits.data(), plan.bits.size() * sizeof(uint32_t), 0},
                     {plan.tile_pages.data(), plan.tile_pages.size() * sizeof(int32_t), 0},
                     {wide.data(), wide.size() * sizeof(int32_t), 0}};
        size_t bytes = 0;
        for (Part& p : parts) {
            p.at = bytes;
            bytes += p.bytes;
        }
        BlockPlanEntry* victim = entry_to_replace(c->block_plans);
        victim->valid = false;
        if (!victim->ev) {
            e = cudaEventCreateWithFlags(&victim->ev, cudaEventDisableTiming);
            if (e != cudaSuccess) return cuda_status(e);
        }
        if (bytes > victim->cap) {
            if (victim->ev_recorded) cudaEventSynchronize(victim->ev);
            if (victim->d) cudaFree(victim->d);
            victim->d = nullptr;
            victim->cap = 0;
            victim->ev_recorded = false;
            const size_t cap = std::max<size_t>(bytes * 5 / 4, 4096);
            e = cudaMalloc(&victim->d, cap);
            if (e != cudaSuccess) {
                cudaGetLastError();
                return cuda_status(e);
            }
            victim->cap = cap;
        }
        if (victim->ev_recorded && victim->ev_stream != st) {
            // the launches that read the old plan run before it is overwritten
            e = cudaStreamWaitEvent(st, victim->ev, 0);
            if (e != cudaSuccess) return cuda_status(e);
        }
        if (c->staging.size() < bytes) c->staging.resize(bytes);
        for (const Part& p : parts)
            if (p.bytes) std::memcpy(c->staging.data() + p.at, p.p, p.bytes);
        rc = staged_copy(c, victim->d, c->staging.data(), bytes, stream);
        if (rc != SQ_OK) return drop_plan(*victim, st, rc);
        victim->tree = parents != nullptr;
        victim->call = std::move(key);
        victim->handles.assign(seqs, seqs + n_seqs);
        victim->versions.resize(n_seqs);
        for (int32_t i = 0; i < n_seqs; ++i) victim->versions[i] = c->host->seq(seqs[i])->version;
        victim->o_items = parts[1].at;
        victim->o_merges = parts[2].at;
        victim->o_rows = plan.rows.empty() ? 0 : parts[3].at;
        victim->o_bits = parts[4].at;
        victim->o_pages = parts[5].at;
        victim->n_words = plan.n_words;
        victim->n_pieces = plan.n_pieces;
        victim->BP = plan.BP;
        victim->n_items = (int32_t)plan.items.size();
        victim->n_merges = (int32_t)plan.merges.size();
        victim->n_parts = plan.n_parts;
        victim->max_splits = plan.max_splits;
        victim->unit_rows = plan.unit_rows;
        victim->one = plan.one;
        victim->n_ctas = plan.n_ctas;
        victim->o_wide = parts[6].at;
        victim->n_wide = (int32_t)wide.size();
        list_writes(c, read.data(), read.size(), &victim->writes);
        victim->valid = true;
        hit = victim;
    } else if (hit->ev_recorded && hit->ev_stream != st) {
        // its upload ran on the stream of the call that planned it
        e = cudaStreamWaitEvent(st, hit->ev, 0);
        if (e != cudaSuccess) return cuda_status(e);
    } else {
        // (a captured launch may run after any work, also work that writes what
        // this one would read ahead of its dependency wait)
        plan_ready = !captured;
    }
    if (captured) keep_captured(c->block_plans, *hit);
    hit->last_use = ++c->use_clock;
    const BlockPlanEntry& plan = *hit;
    if (plan.n_parts > 0 && captured) {
        c->pre_part_captured = true;
    } else if (plan.n_parts > 0) {
        const PrefillPlanEntry* last = c->pre_last;
        if (last && last->ev_recorded && last->ev_stream != st) {
            e = cudaStreamWaitEvent(st, last->ev, 0);
            if (e != cudaSuccess) return drop_plan(*hit, st, cuda_status(e));
        }
        c->pre_last = hit;
    }
    const bool wide = plan.n_wide > 0;
    CUtensorMap qmap, wide_map;
    rc = make_query_map(c, q, (int32_t)n, plan.BP, &qmap);
    if (rc == SQ_OK && wide) rc = widen_pages(c, plan, layer, st, captured, &wide_map);
    if (rc != SQ_OK) return drop_plan(*hit, st, rc);
    BlockShortKv8Args a;
    a.tiles = reinterpret_cast<const PrefillTile*>(plan.d);
    a.items = reinterpret_cast<const PrefillItem*>(plan.d + plan.o_items);
    a.tile_pages = reinterpret_cast<const int32_t*>(plan.d + plan.o_pages);
    a.rows = plan.o_rows ? reinterpret_cast<const int2*>(plan.d + plan.o_rows) : nullptr;
    a.bits = reinterpret_cast<const uint32_t*>(plan.d + plan.o_bits);
    a.n_words = plan.n_words;
    a.pool = wide ? (const void*)c->wide.d : c->pool;
    a.q = q;
    a.n_ctas = plan.n_ctas;
    a.n_pieces = plan.n_pieces;
    a.n_tiles = a.n = a.n_q = 0;  // (the items')
    a.layer = wide ? 0 : layer;
    a.Hq = g.Hq;
    a.Hkv = g.Hkv;
    a.G = g.G();
    a.P = g.P;
    a.num_pages = wide ? plan.n_wide : g.num_pages;
    a.BP = plan.BP;
    a.n_items = plan.n_items;
    a.plan_ready = plan_ready;
    a.n_unsafe = 0;
    a.kv_early = !c->kv8 && plan.one && plan_ready && g.P >= kPrefillKeys / 2 &&
                         early_writes(c, plan.writes, seqs, n_seqs, a.unsafe, &a.n_unsafe)
                     ? 1
                     : 0;
    // (a zero scale as in sq_prefill_attention)
    a.scale_log2 = std::max(sm_scale * 1.4426950408889634f, 1e-30f);
    a.out = out;
    a.out_f32 = out_dtype == SQ_OUT_F32;
    a.lse = lse;
    a.part_o = c->pre_part;
    a.part_ml = c->pre_part ? c->pre_part + (size_t)plan.n_parts * kPrefillQTiles * kPrefillRows * g.D
                            : nullptr;
    a.err = c->d_err;
    a.scales = c->kv8 ? kv8_pool(c).scales : nullptr;
    e = c->kv8 && !wide ? launch_blocks_kv8(c->tmap, qmap, a, g.D, st)
                        : launch_blocks(wide ? wide_map : c->tmap, qmap, a, g.D, plan.one, st);
    if (wide) rc = used_buffer(c->wide, st, captured);
    if (rc != SQ_OK) return drop_plan(*hit, st, rc);
    if (e != cudaSuccess) return drop_plan(*hit, st, cuda_status(e));
    if (plan.n_merges > 0) {
        BlockCombineArgs ca;
        ca.merges = reinterpret_cast<const BlockMerge*>(plan.d + plan.o_merges);
        ca.n_merges = plan.n_merges;
        ca.part_o = a.part_o;
        ca.part_ml = a.part_ml;
        ca.out = out;
        ca.out_f32 = a.out_f32;
        ca.lse = lse;
        ca.Hq = g.Hq;
        ca.G = g.G();
        ca.BP = plan.BP;
        ca.max_splits = plan.max_splits;
        ca.rows = plan.unit_rows;
        e = launch_blocks_combine(ca, g.D, st);
        if (e != cudaSuccess) return drop_plan(*hit, st, cuda_status(e));
    }
    if (!captured) {
        e = cudaEventRecord(hit->ev, st);
        if (e != cudaSuccess) return drop_plan(*hit, st, cuda_status(e));
        hit->ev_recorded = true;
        hit->ev_stream = st;
    }
    for (int32_t i = 0; i < n_seqs; ++i) c->host->seq_mut(seqs[i])->last_stream = stream;
    return SQ_OK;
}

// What of a drafted tree stays.
int accept_impl(sq_cache* c, sq_seq seq, int32_t n_draft, const int32_t* path, int32_t n_path, void* stream) {
    const Seq* s = c->host->seq(seq);
    if (!s) return SQ_ERR_BAD_HANDLE;
    if (n_draft < 0 || n_draft > s->n || n_path < 0 || n_path > n_draft || (n_path > 0 && !path))
        return SQ_ERR_INVALID_ARG;
    for (int32_t i = 0; i < n_path; ++i)
        if (path[i] < 0 || path[i] >= n_draft || (i > 0 && path[i] <= path[i - 1])) return SQ_ERR_INVALID_ARG;
    // the rows between the path's
    const int32_t ctx = s->n - n_draft;
    std::vector<sq_span> spans;
    int32_t next = 0;
    for (int32_t i = 0; i <= n_path; ++i) {
        const int32_t at = i < n_path ? path[i] : n_draft;
        if (at > next) spans.push_back({ctx + next, ctx + at});
        next = at + 1;
    }
    if (spans.empty()) return SQ_OK;
    // packing all of a sequence whose pages are full moves only rows after the
    // first that leaves; of one with partial pages the pages touched are packed
    const int rc =
        evict_impl(c, seq, spans.data(), (int32_t)spans.size(), stream, has_partial_pages(*s, c->g.P));
    if (rc == SQ_OK) c->host->seq_mut(seq)->next_pos -= n_draft - n_path;
    return rc;
}

}  // namespace

extern "C" {

int sq_extend(sq_cache* c, const sq_seq* seqs, int32_t n_seqs, const int32_t* n_new, void* stream) {
    TraceRange trace_("sq_extend");
    if (!c) return SQ_ERR_BAD_HANDLE;
    return guarded([&] { return extend_impl(c, seqs, n_seqs, n_new, stream, nullptr); });
}

int sq_qk_norm_rope_store(sq_cache* c, const sq_seq* seqs, int32_t n_seqs, const int32_t* n_new,
                          int32_t layer, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                          const void* v, int64_t v_stride, const int32_t* positions,
                          const sq_norm_rope* params, void* q_out, void* stream) {
    TraceRange trace_("sq_qk_norm_rope_store");
    if (!c) return SQ_ERR_BAD_HANDLE;
    return guarded([&] {
        return store_impl(c, seqs, n_seqs, n_new, layer, q, q_stride, k, k_stride, v, v_stride, positions,
                          params, q_out, stream);
    });
}

int sq_qk_norm_rope(sq_cache* c, int32_t n_tokens, const void* q, int64_t q_stride, const void* k,
                    int64_t k_stride, const int32_t* positions, const sq_norm_rope* params, void* q_out,
                    void* k_out, void* stream) {
    TraceRange trace_("sq_qk_norm_rope");
    if (!c) return SQ_ERR_BAD_HANDLE;
    return guarded([&] {
        return norm_impl(c, n_tokens, q, q_stride, k, k_stride, positions, params, q_out, k_out, stream);
    });
}

int sq_qk_norm_rope_backward(sq_cache* c, int32_t n_tokens, const void* q, int64_t q_stride, const void* k,
                             int64_t k_stride, const int32_t* positions, const sq_norm_rope* params,
                             const void* dq_out, const void* dk_out, void* dq, int64_t dq_stride, void* dk,
                             int64_t dk_stride, float* dq_weight, float* dk_weight, void* stream) {
    TraceRange trace_("sq_qk_norm_rope_backward");
    if (!c) return SQ_ERR_BAD_HANDLE;
    return guarded([&] {
        return norm_backward_impl(c, n_tokens, q, q_stride, k, k_stride, positions, params, dq_out, dk_out,
                                  dq, dq_stride, dk, dk_stride, dq_weight, dk_weight, stream);
    });
}

int sq_window_attention(sq_cache* c, const sq_seq* seqs, int32_t n_seqs, const int32_t* n_q, int32_t layer,
                        const void* q, void* out, int32_t out_dtype, float* lse, float sm_scale,
                        int32_t window, int32_t n_sink, void* stream) {
    TraceRange trace_("sq_window_attention");
    if (!c) return SQ_ERR_BAD_HANDLE;
    return guarded([&] {
        return blocks_impl(c, seqs, n_seqs, n_q, nullptr, layer, q, out, out_dtype, lse, sm_scale, window,
                           n_sink, stream);
    });
}

int sq_tree_attention(sq_cache* c, const sq_seq* seqs, int32_t n_seqs, const int32_t* n_draft,
                      const int32_t* parents, int32_t layer, const void* q, void* out, int32_t out_dtype,
                      float* lse, float sm_scale, int32_t window, int32_t n_sink, void* stream) {
    TraceRange trace_("sq_tree_attention");
    if (!c) return SQ_ERR_BAD_HANDLE;
    if (n_seqs > 0 && !n_draft) return SQ_ERR_INVALID_ARG;
    static const int32_t none = -1;
    if (!parents) {
        // (only where nothing is drafted)
        for (int32_t i = 0; i < n_seqs; ++i)
            if (n_draft[i] != 0) return SQ_ERR_INVALID_ARG;
        parents = &none;
    }
    return guarded([&] {
        return blocks_impl(c, seqs, n_seqs, n_draft, parents, layer, q, out, out_dtype, lse, sm_scale, window,
                           n_sink, stream);
    });
}

int sq_accept_draft(sq_cache* c, sq_seq seq, int32_t n_draft, const int32_t* path, int32_t n_path,
                    void* stream) {
    TraceRange trace_("sq_accept_draft");
    if (!c) return SQ_ERR_BAD_HANDLE;
    return guarded([&] { return accept_impl(c, seq, n_draft, path, n_path, stream); });
}

}  // extern "C"
