// Calls of caches whose rows are held in 8 bits, and rows read back.  One
// translation unit with sq_api.cpp and operators.inl, whose cache object and helpers
// they share.  See include/sq.h for the contract of every call.

// Rows appended in every layer: n_new[i] of each sequence (null: one), as they are.
static int append_8bit(sq_cache* c, const sq_seq* seqs, int32_t n_seqs, const int32_t* n_new, const void* k,
                       const void* v, void* stream) {
    return guarded([&] {
        if (capturing(as_stream(stream))) return (int)SQ_ERR_UNSUPPORTED;
        int64_t n = 0;
        for (int32_t i = 0; i < n_seqs; ++i) n += n_new ? n_new[i] : 1;
        std::vector<int32_t> pages;
        auto store = [&]() -> int {
            const Geometry& g = c->g;
            cudaStream_t st = as_stream(stream);
            std::vector<RowRun> runs;
            list_runs(c, seqs, n_seqs, n_new, &runs, &pages);
            Kv8StoreInlineArgs a = {};
            a.k = bf16(k);
            a.v = bf16(v);
            a.k_stride = a.v_stride = (int64_t)g.Hkv * g.D;
            a.layer_stride = n * a.k_stride;
            a.pool = kv8_pool(c);
            set_runs(runs, &a);
            a.Hkv = g.Hkv;
            a.n_layers = g.L;
            a.plain = 1;
            a.err = c->d_err;
            int rc;
            if (runs.size() <= (size_t)kRunsInline) {
                std::copy(runs.begin(), runs.end(), a.inline_run);
                rc = cuda_status(launch_kv8_store(a, g.D, st));
            } else {
                rc = with_upload(c, runs.data(), runs.size() * sizeof(RowRun), stream, [&](const uint8_t* d) {
                    a.runs = reinterpret_cast<const RowRun*>(d);
                    return launch_kv8_store(a, g.D, st);
                });
            }
            if (rc == SQ_OK) note_writes(c, pages.data(), pages.size(), stream);
            return rc;
        };
        return extend_impl(c, seqs, n_seqs, n_new, stream, store);
    });
}

namespace {

int read_impl(sq_cache* c, const sq_seq* seqs, int32_t n_seqs, const int32_t* counts, int32_t layer, void* k,
              void* v, void* stream) {
    if (!launch_kv8_read) return SQ_ERR_UNSUPPORTED;
    const Geometry& g = c->g;
    int64_t n = 0;
    int rc = check_handles(c, seqs, n_seqs);
    if (rc == SQ_OK) rc = check_counts(c, seqs, n_seqs, counts, &n);
    if (rc != SQ_OK) return rc;
    if (layer < 0 || layer >= g.L) return SQ_ERR_INVALID_ARG;
    if (n == 0) return SQ_OK;
    const int64_t w = (int64_t)g.Hkv * g.D;
    if (!rows_ok(k, w, w) || !rows_ok(v, w, w)) return SQ_ERR_INVALID_ARG;
    if (any_overlap({{c->pool, c->pool_bytes}}, {{k, rows_bytes(n, w, w)}, {v, rows_bytes(n, w, w)}}))
        return SQ_ERR_INVALID_ARG;
    std::vector<RowRun> runs;
    list_runs(c, seqs, n_seqs, counts, &runs, nullptr);
    cudaStream_t st = as_stream(stream);
    Kv8ReadInlineArgs a;
    a.pool = {nullptr, nullptr, g.num_pages, g.Hkv, g.P};
    if (c->kv8) a.pool = kv8_pool(c);
    a.wide = c->kv8 ? nullptr : c->pool;
    a.runs = nullptr;
    a.k = bf16(k);
    a.v = bf16(v);
    a.n_runs = (int32_t)runs.size();
    a.most = 0;
    for (const RowRun& r : runs) a.most = std::max(a.most, r.n);
    a.layer = layer;
    a.err = c->d_err;
    if (runs.size() <= (size_t)kRunsInline) {
        std::copy(runs.begin(), runs.end(), a.inline_run);
        rc = cuda_status(launch_kv8_read(a, g.D, st));
    } else if (capturing(st)) {
        rc = SQ_ERR_UNSUPPORTED;
    } else {
        rc = with_upload(c, runs.data(), runs.size() * sizeof(RowRun), stream, [&](const uint8_t* d) {
            a.runs = reinterpret_cast<const RowRun*>(d);
            return launch_kv8_read(a, g.D, st);
        });
    }
    if (rc != SQ_OK) return rc;
    for (int32_t i = 0; i < n_seqs; ++i) c->host->seq_mut(seqs[i])->last_stream = stream;
    return SQ_OK;
}

}  // namespace

extern "C" {

int sq_read_kv(sq_cache* c, const sq_seq* seqs, int32_t n_seqs, const int32_t* counts, int32_t layer, void* k,
               void* v, void* stream) {
    TraceRange trace_("sq_read_kv");
    if (!c) return SQ_ERR_BAD_HANDLE;
    return guarded([&] { return read_impl(c, seqs, n_seqs, counts, layer, k, v, stream); });
}

}  // extern "C"
