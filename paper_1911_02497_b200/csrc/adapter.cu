// Host side of the low-rank adapters: argument checks, tiles and splits, launches.
#include <cmath>
#include <cstddef>
#include <new>

#include "adapter.cuh"
#include "ctx.cuh"

using namespace cs;

static_assert(CONDENSA_ADAPTER_MAX_RANK == AD_MAX_RANK, "largest rank");

namespace {

struct Run {
    int first, count;               // rows
};

// The rows of a batch by adapter.
struct Rows {
    long long total = 0, live = 0;              // rows of the batch; rows with an adapter
    std::vector<int> used;                      // adapters with rows, ascending
    std::vector<std::vector<Run>> runs;         // of used[i]
    int max_rank = 0;
};

struct Tiles {
    std::vector<AdapterTile> tile;              // `list` into `rows`
    std::vector<int> owner;                     // place in Rows::used
    std::vector<int> rows;
};

int type_bytes(int dtype) { return dtype == CONDENSA_DTYPE_FP32 ? 4 : 2; }

// Widest access (16, 8, 4, 2 bytes) that a row start of `p` with rows `stride` bytes apart allows.
int widest(const void *p, long long stride)
{
    const uintptr_t bits = (uintptr_t)p | (uintptr_t)stride;
    return bits % 16 == 0 ? 16 : bits % 8 == 0 ? 8 : bits % 4 == 0 ? 4 : 2;
}

int read_batch(condensa_ctx *ctx, const condensa_adapter_batch *b, Rows &rows)
{
    if (!b) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "batch is NULL");
    if (b->dtype != CONDENSA_DTYPE_FP32 && b->dtype != CONDENSA_DTYPE_FP16 && b->dtype != CONDENSA_DTYPE_BF16)
        return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "dtype must be CONDENSA_DTYPE_FP32, _FP16 or _BF16");
    if (b->reserved != 0) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "reserved must be 0");
    if (b->n_adapters < 0 || (b->n_adapters > 0 && !b->adapters)) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "adapters is NULL");
    if (b->n_requests < 0 || (b->n_requests > 0 && (!b->request_rows || !b->request_adapter)))
        return fail(ctx, CONDENSA_ERR_INVALID_ARG, "request lists are NULL");
    if (b->k < 1 || b->n < 1) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "k and n must be positive");
    if (b->k > 0x7FFFFFFFll || b->n > 0x7FFFFFFFll) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "k and n must be below 2^31");
    std::vector<int> place((size_t)b->n_adapters, -1);
    for (int q = 0; q < b->n_requests; ++q) {
        const long long n = b->request_rows[q];
        const int a = b->request_adapter[q];
        if (n < 0) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "request %d: negative rows", q);
        if (a < -1 || a >= b->n_adapters) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "request %d: no adapter %d", q, a);
        if (n > 0x7FFFFFFFll - rows.total) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "a batch has fewer than 2^31 rows");
        if (n > 0 && a >= 0) {
            rows.live += n;
            place[a] = 0;
        }
        rows.total += n;
    }
    for (int a = 0; a < b->n_adapters; ++a) {
        if (place[a] < 0) continue;
        const condensa_adapter &x = b->adapters[a];
        if (!x.a || !x.b) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "adapter %d: a or b is NULL", a);
        place[a] = (int)rows.used.size();
        rows.used.push_back(a);
    }
    const int e = type_bytes(b->dtype);
    for (int a = 0; a < b->n_adapters; ++a) {
        const condensa_adapter &x = b->adapters[a];
        const bool grads = x.grad_a || x.grad_b;
        if (place[a] < 0 && !grads) continue;
        if (x.rank < 1) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "adapter %d: rank must be positive", a);
        if (x.rank > AD_MAX_RANK) return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "adapter %d: ranks above %d are not built", a, AD_MAX_RANK);
        if (!std::isfinite(x.scale)) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "adapter %d: scale must be finite", a);
        if ((uintptr_t)x.a % e || (uintptr_t)x.b % e || (uintptr_t)x.grad_a % 4 || (uintptr_t)x.grad_b % 4)
            return fail(ctx, CONDENSA_ERR_INVALID_ARG, "adapter %d: a pointer is not aligned to its type", a);
        if (place[a] >= 0) rows.max_rank = std::max(rows.max_rank, (int)x.rank);
    }
    rows.runs.resize(rows.used.size());
    int at = 0;
    for (int q = 0; q < b->n_requests; ++q) {
        const int n = (int)b->request_rows[q], a = b->request_adapter[q];
        if (n > 0 && a >= 0) {
            std::vector<Run> &r = rows.runs[(size_t)place[a]];
            if (!r.empty() && r.back().first + r.back().count == at) r.back().count += n;
            else r.push_back({at, n});
        }
        at += n;
    }
    return CONDENSA_OK;
}

// Cuts every adapter's rows into tiles of up to `tm`.
void make_tiles(const Rows &rows, int tm, Tiles &t)
{
    std::vector<Run> part;
    for (size_t a = 0; a < rows.used.size(); ++a) {
        int filled = 0;
        part.clear();
        auto flush = [&]() {
            if (!filled) return;
            AdapterTile x;
            x.first = part[0].first;
            x.count = (u16)filled;
            x.adapter = (u16)0;
            x.list = -1;
            if (part.size() > 1) {
                x.list = (int)t.rows.size();
                for (const Run &r : part)
                    for (int i = 0; i < r.count; ++i) t.rows.push_back(r.first + i);
            }
            t.tile.push_back(x);
            t.owner.push_back((int)a);
            filled = 0;
            part.clear();
        };
        for (const Run &r : rows.runs[a]) {
            for (int done = 0; done < r.count;) {
                const int n = std::min(r.count - done, tm - filled);
                part.push_back({r.first + done, n});
                filled += n;
                done += n;
                if (filled == tm) flush();
            }
        }
        flush();
    }
}

// The tiles of one launch, as they go into its parameters.
struct TileList {
    std::vector<AdapterTile> tiles;
    std::vector<int> rows;
    size_t bytes() const { return tiles.size() * sizeof(AdapterTile) + rows.size() * sizeof(int); }
    size_t bytes_with(const AdapterTile &x) const { return bytes() + sizeof(AdapterTile) + (x.list >= 0 ? x.count * sizeof(int) : 0); }
    void add(const Tiles &t, size_t i, int entry)
    {
        AdapterTile x = t.tile[i];
        if (x.list >= 0) {
            const int from = x.list;
            x.list = (int)rows.size();
            rows.insert(rows.end(), t.rows.begin() + from, t.rows.begin() + from + x.count);
        }
        x.adapter = (u16)entry;
        tiles.push_back(x);
    }
    void write(char *p) const
    {
        if (!tiles.empty()) memcpy(p, tiles.data(), tiles.size() * sizeof(AdapterTile));
        if (!rows.empty()) memcpy(p + tiles.size() * sizeof(AdapterTile), rows.data(), rows.size() * sizeof(int));
    }
};

// ------------------------------------------------------------------ kernels by type, tile height, rank
template <class T, bool TRANS, int TM, int RP>
int launch_adapter_of(condensa_ctx *ctx, const AdapterParams &P, int cluster, int id, cudaStream_t stream)
{
    using G = AdGeom<T, TRANS, TM, RP>;
    const void *kernel = (const void *)k_adapter<T, TRANS, TM, RP>;
    if (!(ctx->op_smem_set >> id & 1)) {
        CU_TRY(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, G::SMEM));
        ctx->op_smem_set |= 1ull << id;
    }
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)(P.n_tiles * cluster));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = G::SMEM;
    cfg.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)cluster;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    const int pa_ = prof_begin(ctx, TRANS ? "k_adapter_backward" : "k_adapter_forward", stream);
    void *args[] = {(void *)&P};
    CU_TRY(ctx, cudaLaunchKernelExC(&cfg, kernel, args));
    ctx->launches += 1;
    prof_end(ctx, pa_, stream);
    return CONDENSA_OK;
}

template <class T, bool TRANS, int TM>
int launch_adapter_rank(condensa_ctx *ctx, const AdapterParams &P, int cluster, int rank, int id, cudaStream_t stream)
{
    if (rank <= 16) return launch_adapter_of<T, TRANS, TM, 16>(ctx, P, cluster, id, stream);
    if (rank <= 32) return launch_adapter_of<T, TRANS, TM, 32>(ctx, P, cluster, id + 1, stream);
    if (rank <= 64) return launch_adapter_of<T, TRANS, TM, 64>(ctx, P, cluster, id + 2, stream);
    return launch_adapter_of<T, TRANS, TM, 128>(ctx, P, cluster, id + 3, stream);
}

template <class T>
int launch_adapter_type(condensa_ctx *ctx, const AdapterParams &P, bool trans, int tm, int cluster, int rank, int id, cudaStream_t stream)
{
    if (!trans) return tm == 16 ? launch_adapter_rank<T, false, 16>(ctx, P, cluster, rank, id, stream) : launch_adapter_rank<T, false, 64>(ctx, P, cluster, rank, id + 4, stream);
    return tm == 16 ? launch_adapter_rank<T, true, 16>(ctx, P, cluster, rank, id + 8, stream) : launch_adapter_rank<T, true, 64>(ctx, P, cluster, rank, id + 12, stream);
}

int launch_adapter(condensa_ctx *ctx, const AdapterParams &P, int dtype, bool trans, int tm, int cluster, int rank, cudaStream_t stream)
{
    if (dtype == CONDENSA_DTYPE_BF16) return launch_adapter_type<__nv_bfloat16>(ctx, P, trans, tm, cluster, rank, 0, stream);
    if (dtype == CONDENSA_DTYPE_FP16) return launch_adapter_type<__half>(ctx, P, trans, tm, cluster, rank, 16, stream);
    return launch_adapter_type<float>(ctx, P, trans, tm, cluster, rank, 32, stream);
}

template <class T, int RP>
int launch_wgrad_of(condensa_ctx *ctx, WgradParams &P, int id, cudaStream_t stream)
{
    using G = WgGeom<T, RP>;
    const void *kernel = (const void *)k_adapter_wgrad<T, RP>;
    if (!(ctx->op_smem_set >> id & 1)) {
        CU_TRY(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, G::SMEM));
        ctx->op_smem_set |= 1ull << id;
    }
    P.strips0 = (int)((P.side[0].width + G::WC - 1) / G::WC);
    const int strips1 = (int)((P.side[1].width + G::WC - 1) / G::WC);
    const int pa_ = prof_begin(ctx, "k_adapter_wgrad", stream);
    k_adapter_wgrad<T, RP><<<dim3((unsigned)(P.strips0 + strips1), (unsigned)P.n_splits), THREADS, G::SMEM, stream>>>(P);
    LAUNCH_CHECK(ctx);
    prof_end(ctx, pa_, stream);
    return CONDENSA_OK;
}

template <class T>
int launch_wgrad_type(condensa_ctx *ctx, WgradParams &P, int rank, int id, cudaStream_t stream)
{
    if (rank <= 16) return launch_wgrad_of<T, 16>(ctx, P, id, stream);
    if (rank <= 32) return launch_wgrad_of<T, 32>(ctx, P, id + 1, stream);
    if (rank <= 64) return launch_wgrad_of<T, 64>(ctx, P, id + 2, stream);
    return launch_wgrad_of<T, 128>(ctx, P, id + 3, stream);
}

int wgrad_strip(int dtype, int rank) { return dtype != CONDENSA_DTYPE_FP32 && rank <= 64 ? WgGeom<__half, 64>::WC : WgGeom<float, 64>::WC; }

// ------------------------------------------------------------------ both directions of the row kernel
struct RowCall {
    const void *src;
    void *dst;
    float *h;
    long long ld_src, ld_dst, ld_h;
    bool trans;
};

int run_rows(condensa_ctx *ctx, const condensa_adapter_batch *b, const Rows &rows, const RowCall &c, cudaStream_t stream)
{
    const int e = type_bytes(b->dtype);
    const long long ws = c.trans ? b->n : b->k, wd = c.trans ? b->k : b->n;
    // tiles of 64 rows where the adapters have that many; for a few rows each, 16 waste less and spread further
    const int tm = rows.live >= 48ll * (long long)rows.used.size() ? 64 : 16;
    Tiles t;
    make_tiles(rows, tm, t);
    // as many CTAs per tile as it takes to cover the SMs about twice
    int cluster = 1;
    while (cluster < AD_MAX_CLUSTER && (long long)t.tile.size() * cluster < 2ll * ctx->num_sms) cluster *= 2;
    AdapterParams P;
    P.src = c.src; P.dst = c.dst; P.h = c.h;
    P.ld_src = c.ld_src; P.ld_dst = c.ld_dst; P.ld_h = c.ld_h;
    P.width_src = ws; P.width_dst = wd;
    P.vec_src = widest(c.src, c.ld_src * e);
    P.vec_dst = c.dst ? widest(c.dst, c.ld_dst * e) : 16;
    for (size_t i = 0; i < t.tile.size();) {        // as many tiles per launch as their lists fit the parameters
        std::vector<AdapterEntry> entries;
        TileList l;
        for (int last = -1; i < t.tile.size(); ++i) {
            const int a = t.owner[i];
            if ((entries.size() + (a != last)) * sizeof(AdapterEntry) + l.bytes_with(t.tile[i]) > AD_BLOB) break;
            if (a != last) {
                const condensa_adapter &ad = b->adapters[rows.used[a]];
                const uint8_t va = (uint8_t)widest(ad.a, b->k * e), vb = (uint8_t)widest(ad.b, (long long)ad.rank * e);
                AdapterEntry en;
                en.shrink = c.trans ? ad.b : ad.a;
                en.expand = c.trans ? ad.a : ad.b;
                en.scale = ad.scale;
                en.rank = (u16)ad.rank;
                en.vec_s = c.trans ? vb : va;
                en.vec_e = c.trans ? va : vb;
                entries.push_back(en);
                last = a;
            }
            l.add(t, i, (int)entries.size() - 1);
        }
        P.n_entries = (int)entries.size();
        P.n_tiles = (int)l.tiles.size();
        char *p = (char *)P.blob;
        memcpy(p, entries.data(), entries.size() * sizeof(AdapterEntry));
        l.write(p + entries.size() * sizeof(AdapterEntry));
        const int rc = launch_adapter(ctx, P, b->dtype, c.trans, tm, cluster, rows.max_rank, stream);
        if (rc) return rc;
    }
    return CONDENSA_OK;
}

// ------------------------------------------------------------------ weight gradients
struct Split {
    int owner, tile0, n_tiles;
};

struct Wgrad {
    const void *x, *dy;
    const float *u, *h;
    long long ldx, lddy, ldu, ldh;
    bool need_a, need_b;                // some adapter has a grad_a, a grad_b
    int accumulate;
};

// Splits of the adapters' rows, and the workspace that their sums take (floats).
void make_splits(const condensa_ctx *ctx, const condensa_adapter_batch *b, const Rows &rows, const Tiles &t, std::vector<Split> &splits,
                 std::vector<long long> &slot, long long &floats)
{
    const int wc = wgrad_strip(b->dtype, rows.max_rank);
    const long long strips = (b->k + wc - 1) / wc + (b->n + wc - 1) / wc;
    // CTAs for about four rounds of the SMs; a split's sums are written and read again, so none is shorter than four tiles
    const long long want = std::max<long long>(1, 4ll * ctx->num_sms / strips);
    const int per = (int)std::min<long long>(0x7FFF, std::max<long long>(4, ((long long)t.tile.size() + want - 1) / want));
    std::vector<int> count(rows.used.size(), 0);
    TileList l;
    for (size_t i = 0; i < t.tile.size(); ++i) {
        const bool fits = sizeof(WgEntry) + sizeof(WgSplit) + l.bytes_with(t.tile[i]) <= AD_BLOB;
        if (splits.empty() || splits.back().owner != t.owner[i] || splits.back().n_tiles == per || !fits) {
            splits.push_back({t.owner[i], (int)i, 0});
            count[t.owner[i]] += 1;
            l = TileList();
        }
        splits.back().n_tiles += 1;
        l.add(t, i, 0);
    }
    floats = 0;
    slot.assign(rows.used.size(), -1);
    for (size_t a = 0; a < rows.used.size(); ++a) {
        if (count[a] <= 1) continue;
        slot[a] = floats;
        floats += (long long)count[a] * b->adapters[rows.used[a]].rank * (b->k + b->n);
    }
}

int run_wgrad(condensa_ctx *ctx, const condensa_adapter_batch *b, const Rows &rows, const Tiles &t, const std::vector<Split> &splits,
              const std::vector<long long> &slot, const Wgrad &w, float *part, cudaStream_t stream)
{
    const int e = type_bytes(b->dtype);
    WgradParams P;
    memset(&P, 0, offsetof(WgradParams, blob));
    P.side[0] = {w.x, w.u, w.ldx, w.ldu, b->k, w.x ? widest(w.x, w.ldx * e) : 16, w.u ? widest(w.u, w.ldu * 4) : 16};
    P.side[1] = {w.dy, w.h, w.lddy, w.ldh, b->n, widest(w.dy, w.lddy * e), w.h ? widest(w.h, w.ldh * 4) : 16};
    P.part = part;
    P.accumulate = w.accumulate;
    std::vector<int> of_owner(rows.used.size(), 0);         // splits of an adapter so far
    for (size_t i = 0; i < splits.size();) {
        std::vector<WgEntry> entries;
        std::vector<WgSplit> sp;
        TileList l;
        for (int last = -1; i < splits.size(); ++i) {
            const Split &q = splits[i];
            const condensa_adapter &ad = b->adapters[rows.used[q.owner]];
            size_t bytes = (entries.size() + (q.owner != last)) * sizeof(WgEntry) + (sp.size() + 1) * sizeof(WgSplit);
            TileList with = l;
            for (int k = 0; k < q.n_tiles; ++k) with.add(t, (size_t)(q.tile0 + k), 0);
            if (!sp.empty() && bytes + with.bytes() > AD_BLOB) break;
            if (q.owner != last) {
                entries.push_back({{ad.grad_a, ad.grad_b}, ad.scale, ad.rank});
                last = q.owner;
            }
            WgSplit x;
            x.slot = slot[q.owner] < 0 ? -1 : slot[q.owner] + (long long)of_owner[q.owner] * ad.rank * (b->k + b->n);
            x.tile0 = (int)l.tiles.size();
            x.n_tiles = (u16)q.n_tiles;
            x.adapter = (u16)(entries.size() - 1);
            of_owner[q.owner] += 1;
            sp.push_back(x);
            l = with;
        }
        P.n_entries = (int)entries.size();
        P.n_splits = (int)sp.size();
        P.n_tiles = (int)l.tiles.size();
        char *p = (char *)P.blob;
        memcpy(p, entries.data(), entries.size() * sizeof(WgEntry)); p += entries.size() * sizeof(WgEntry);
        memcpy(p, sp.data(), sp.size() * sizeof(WgSplit)); p += sp.size() * sizeof(WgSplit);
        l.write(p);
        int rc;
        if (b->dtype == CONDENSA_DTYPE_BF16) rc = launch_wgrad_type<__nv_bfloat16>(ctx, P, rows.max_rank, 48, stream);
        else if (b->dtype == CONDENSA_DTYPE_FP16) rc = launch_wgrad_type<__half>(ctx, P, rows.max_rank, 52, stream);
        else rc = launch_wgrad_type<float>(ctx, P, rows.max_rank, 56, stream);
        if (rc) return rc;
    }
    // gradients of several splits, and of adapters without rows (zeros, or nothing to add)
    ReduceParams R;
    memset(&R, 0, offsetof(ReduceParams, e));
    R.part = part;
    R.width[0] = b->k;
    R.width[1] = b->n;
    R.accumulate = w.accumulate;
    int n = 0;
    long long most = 0;
    auto flush = [&]() -> int {
        if (!n) return CONDENSA_OK;
        const int blocks = (int)std::min<long long>((most + THREADS - 1) / THREADS, 4ll * ctx->num_sms);
        const int pa_ = prof_begin(ctx, "k_adapter_reduce", stream);
        k_adapter_reduce<<<dim3((unsigned)blocks, (unsigned)n), THREADS, 0, stream>>>(R);
        LAUNCH_CHECK(ctx);
        prof_end(ctx, pa_, stream);
        n = 0;
        most = 0;
        return CONDENSA_OK;
    };
    size_t u = 0;
    for (int a = 0; a < b->n_adapters; ++a) {
        const condensa_adapter &ad = b->adapters[a];
        const bool live = u < rows.used.size() && rows.used[u] == a;
        const size_t owner = u;
        if (live) ++u;
        if (!ad.grad_a && !ad.grad_b) continue;
        if (live ? slot[owner] < 0 : w.accumulate != 0) continue;
        R.e[n++] = {{ad.grad_a, ad.grad_b}, live ? slot[owner] : 0, live ? of_owner[owner] : 0, ad.rank};
        most = std::max(most, (long long)ad.rank * (b->k + b->n));
        if (n == AD_RED_MAX) {
            const int rc = flush();
            if (rc) return rc;
        }
    }
    return flush();
}

// ------------------------------------------------------------------ calls
struct Ranges {
    std::vector<Interval> iv;
    void add(const void *p, long long bytes, bool out)
    {
        if (p && bytes > 0) iv.push_back({(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, out});
    }
};

// A matrix of `rows` x `width` values: checked, and its range noted.
int take_rows(condensa_ctx *ctx, const char *name, const void *p, long long ld, long long rows, long long width, int e, bool out, Ranges &r)
{
    if (rows == 0) return CONDENSA_OK;
    if (!p) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "%s is NULL", name);
    if ((uintptr_t)p % e) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "%s is not aligned to its type", name);
    if (ld < width) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "%s: rows of %lld values lie %lld apart", name, width, ld);
    if (ld > (1ll << 40)) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "%s: row stride above 2^40", name);
    r.add(p, ((rows - 1) * ld + width) * e, out);
    return CONDENSA_OK;
}

int forward(condensa_ctx *ctx, const condensa_adapter_batch *b, const void *x, long long ldx, void *y, long long ldy, float *h, long long ldh,
            cudaStream_t stream)
{
    Rows rows;
    int rc = read_batch(ctx, b, rows);
    if (rc) return rc;
    const int e = type_bytes(b->dtype);
    Ranges r;
    if ((rc = take_rows(ctx, "x", x, ldx, rows.total, b->k, e, false, r)) != 0) return rc;
    if ((rc = take_rows(ctx, "y", y, ldy, rows.total, b->n, e, true, r)) != 0) return rc;
    if (h && (rc = take_rows(ctx, "h", h, ldh, rows.total, rows.max_rank, 4, true, r)) != 0) return rc;
    for (int a : rows.used) {
        const condensa_adapter &ad = b->adapters[a];
        r.add(ad.a, (long long)ad.rank * b->k * e, false);
        r.add(ad.b, (long long)ad.rank * b->n * e, false);
    }
    if (ranges_clash(r.iv)) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "an output buffer overlaps another buffer of the call");
    if (rows.live == 0) return CONDENSA_OK;
    CU_TRY(ctx, cudaSetDevice(ctx->device));
    return run_rows(ctx, b, rows, {x, y, h, ldx, ldy, ldh, false}, stream);
}

int backward(condensa_ctx *ctx, const condensa_adapter_batch *b, const void *x, long long ldx, const void *dy, long long lddy, const float *h,
             long long ldh, void *dx, long long lddx, int accumulate, cudaStream_t stream)
{
    Rows rows;
    int rc = read_batch(ctx, b, rows);
    if (rc) return rc;
    const int e = type_bytes(b->dtype);
    bool need_a = false, need_b = false, any = false;       // of adapters with rows; of any adapter
    for (int a : rows.used) {
        need_a = need_a || b->adapters[a].grad_a;
        need_b = need_b || b->adapters[a].grad_b;
    }
    Ranges r;
    if ((rc = take_rows(ctx, "dy", dy, lddy, rows.total, b->n, e, false, r)) != 0) return rc;
    if (dx && (rc = take_rows(ctx, "dx", dx, lddx, rows.total, b->k, e, true, r)) != 0) return rc;
    if (need_a && (rc = take_rows(ctx, "x", x, ldx, rows.total, b->k, e, false, r)) != 0) return rc;
    if (need_b && (rc = take_rows(ctx, "h", h, ldh, rows.total, rows.max_rank, 4, false, r)) != 0) return rc;
    size_t u = 0;
    for (int a = 0; a < b->n_adapters; ++a) {
        const condensa_adapter &ad = b->adapters[a];
        if (u < rows.used.size() && rows.used[u] == a) {
            ++u;
            r.add(ad.a, (long long)ad.rank * b->k * e, false);
            r.add(ad.b, (long long)ad.rank * b->n * e, false);
        }
        any = any || ad.grad_a || ad.grad_b;
        r.add(ad.grad_a, (long long)ad.rank * b->k * 4, true);
        r.add(ad.grad_b, (long long)ad.rank * b->n * 4, true);
    }
    if (ranges_clash(r.iv)) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "an output buffer overlaps another buffer of the call");
    CU_TRY(ctx, cudaSetDevice(ctx->device));
    if (!any) return rows.live && dx ? run_rows(ctx, b, rows, {dy, dx, nullptr, lddy, lddx, 0, true}, stream) : CONDENSA_OK;
    Tiles t;
    make_tiles(rows, AD_WG_ROWS, t);
    std::vector<Split> splits;
    std::vector<long long> slot;
    long long floats = 0;
    if (need_a || need_b) make_splits(ctx, b, rows, t, splits, slot, floats);
    else slot.assign(rows.used.size(), -1);
    const long long ldu = (rows.max_rank + 3) / 4 * 4;
    const size_t u_bytes = need_a ? align_up(sizeof(float) * (size_t)(rows.total * ldu), 256) : 0;
    rc = op_workspace(ctx, 256 + u_bytes + sizeof(float) * (size_t)floats, stream);
    if (rc) return rc;
    float *u_ws = need_a ? (float *)(ctx->op_ws + 256) : nullptr;
    float *part = (float *)(ctx->op_ws + 256 + u_bytes);
    if (rows.live && (dx || need_a) && (rc = run_rows(ctx, b, rows, {dy, dx, u_ws, lddy, lddx, ldu, true}, stream)) != 0) return rc;
    rc = run_wgrad(ctx, b, rows, t, splits, slot, {x, dy, u_ws, h, ldx, lddy, ldu, ldh, need_a, need_b, accumulate != 0}, part, stream);
    if (rc) return rc;
    return op_workspace_done(ctx, stream);
}

}  // namespace

extern "C" {

int condensa_adapter_forward(condensa_ctx *ctx, const condensa_adapter_batch *batch, const void *x, int64_t ldx, void *y, int64_t ldy, float *h,
                             int64_t ldh, void *stream)
{
    if (!ctx) return CONDENSA_ERR_INVALID_ARG;
    try {
        return forward(ctx, batch, x, ldx, y, ldy, h, ldh, (cudaStream_t)stream);
    } catch (const std::bad_alloc &) {
        return fail(ctx, CONDENSA_ERR_WORKSPACE, "out of host memory");
    }
}

int condensa_adapter_backward(condensa_ctx *ctx, const condensa_adapter_batch *batch, const void *x, int64_t ldx, const void *dy, int64_t lddy,
                              const float *h, int64_t ldh, void *dx, int64_t lddx, int accumulate, void *stream)
{
    if (!ctx) return CONDENSA_ERR_INVALID_ARG;
    try {
        return backward(ctx, batch, x, ldx, dy, lddy, h, ldh, dx, lddx, accumulate, (cudaStream_t)stream);
    } catch (const std::bad_alloc &) {
        return fail(ctx, CONDENSA_ERR_WORKSPACE, "out of host memory");
    }
}

}  // extern "C"
