// Host side of the low-rank adapters: argument checks, rows by adapter, launches.
#include <cmath>
#include <cstddef>
#include <new>

#include "adapter_launch.cuh"

using namespace cs;

static_assert(CONDENSA_ADAPTER_MAX_RANK == AD_MAX_RANK, "largest rank");
static_assert(AD_WG_ROWS <= 64, "rows of a tile, in the limit of a batch");

namespace {

struct Run {
    int first, count;               // rows that follow one another
};

// The rows of a batch by adapter.
struct Rows {
    long long total = 0, live = 0;              // rows of the batch; rows with an adapter
    std::vector<int> used;                      // adapters with rows, ascending
    std::vector<int> begin;                     // used[i]'s runs: [begin[i], end[i])
    std::vector<int> end;
    std::vector<int> count;                     // rows of used[i]
    std::vector<Run> runs;
    int max_rank = 0;
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
    if (b->k > AD_MAX_WIDTH || b->n > AD_MAX_WIDTH) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "k and n must not exceed %d", AD_MAX_WIDTH);
    std::vector<int> place((size_t)b->n_adapters, 0);          // requests with rows, then the place in `used`
    int live_requests = 0;
    for (int q = 0; q < b->n_requests; ++q) {
        const long long n = b->request_rows[q];
        const int a = b->request_adapter[q];
        if (n < 0) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "request %d: negative rows", q);
        if (a < -1 || a >= b->n_adapters) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "request %d: no adapter %d", q, a);
        // (a tile's rows are counted in 32 bits past the last one)
        if (n > (1ll << 31) - 64 - rows.total) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "a batch has at most 2^31 - 64 rows");
        if (n > 0 && a >= 0) {
            rows.live += n;
            place[a] += 1;
            ++live_requests;
        }
        rows.total += n;
    }
    if (rows.total != b->rows) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "the requests have %lld rows, the batch %lld", rows.total, (long long)b->rows);
    const int e = type_bytes(b->dtype);
    int at = 0;
    for (int a = 0; a < b->n_adapters; ++a) {
        const condensa_adapter &x = b->adapters[a];
        const bool live = place[a] > 0;
        if (!live && !x.grad_a && !x.grad_b) continue;
        if (live && (!x.a || !x.b)) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "adapter %d: a or b is NULL", a);
        if (x.rank < 1) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "adapter %d: rank must be positive", a);
        if (x.rank > AD_MAX_RANK) return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "adapter %d: ranks above %d are not built", a, AD_MAX_RANK);
        if (!std::isfinite(x.scale)) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "adapter %d: scale must be finite", a);
        if ((uintptr_t)x.a % e || (uintptr_t)x.b % e || (uintptr_t)x.grad_a % 4 || (uintptr_t)x.grad_b % 4)
            return fail(ctx, CONDENSA_ERR_INVALID_ARG, "adapter %d: a pointer is not aligned to its type", a);
        if (!live) continue;
        rows.max_rank = std::max(rows.max_rank, (int)x.rank);
        rows.begin.push_back(at);
        at += place[a];
        place[a] = (int)rows.used.size();
        rows.used.push_back(a);
    }
    rows.end = rows.begin;
    rows.count.assign(rows.used.size(), 0);
    rows.runs.resize((size_t)live_requests);
    int first = 0;
    for (int q = 0; q < b->n_requests; ++q) {
        const int n = (int)b->request_rows[q], a = b->request_adapter[q];
        if (n > 0 && a >= 0) {
            const int i = place[a];
            Run *last = rows.end[i] > rows.begin[i] ? &rows.runs[rows.end[i] - 1] : nullptr;
            if (last && last->first + last->count == first) last->count += n;
            else rows.runs[rows.end[i]++] = {first, n};
            rows.count[i] += n;
        }
        first += n;
    }
    return CONDENSA_OK;
}

// Entries of the adapters and their runs, as they go into the parameters of a launch.
template <class Entry>
struct Blob {
    std::vector<Entry> entries;
    std::vector<AdapterRun> runs;
    int room() const { return (int)((AD_BLOB - (entries.size() + 1) * sizeof(Entry)) / sizeof(AdapterRun)) - (int)runs.size(); }
    // Adds runs [from, to) of the batch for `e`.
    void add(Entry e, const Rows &rows, int from, int to)
    {
        e.run0 = (u16)runs.size();
        e.n_runs = (u16)(to - from);
        e.n_rows = 0;
        for (int r = from; r < to; ++r) {
            runs.push_back({rows.runs[r].first, e.n_rows});
            e.n_rows += rows.runs[r].count;
        }
        entries.push_back(e);
    }
    void write(u32 *blob) const
    {
        char *p = (char *)blob;
        if (!entries.empty()) memcpy(p, entries.data(), entries.size() * sizeof(Entry));
        if (!runs.empty()) memcpy(p + entries.size() * sizeof(Entry), runs.data(), runs.size() * sizeof(AdapterRun));
    }
    void clear()
    {
        entries.clear();
        runs.clear();
    }
};

// ------------------------------------------------------------------ launches
int allow_smem(condensa_ctx *ctx, const AdapterKernel &k)
{
    for (const void *f : ctx->op_smem_set)
        if (f == k.f) return CONDENSA_OK;
    CU_TRY(ctx, cudaFuncSetAttribute(k.f, cudaFuncAttributeMaxDynamicSharedMemorySize, k.smem));
    ctx->op_smem_set.push_back(k.f);
    return CONDENSA_OK;
}

// A launch in clusters; `pdl`: it may start while the kernel ahead of it ends.
int launch_cluster(condensa_ctx *ctx, const AdapterKernel &k, dim3 grid, dim3 cluster, bool pdl, void *params, const char *name, cudaStream_t stream)
{
    const int rc = allow_smem(ctx, k);
    if (rc) return rc;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)k.threads);
    cfg.dynamicSmemBytes = (size_t)k.smem;
    cfg.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = cluster.x;
    at[0].val.clusterDim.y = cluster.y;
    at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = pdl && !ctx->prof_on ? 2 : 1;
    void *args[] = {params};
    const int pa_ = prof_begin(ctx, name, stream);
    CU_TRY(ctx, cudaLaunchKernelExC(&cfg, k.f, args));
    ctx->launches += 1;
    prof_end(ctx, pa_, stream);
    return CONDENSA_OK;
}

// Clusters of `n` CTAs of a kernel that the device holds at once (clusters do not cross its groups of SMs).
int resident_clusters(condensa_ctx *ctx, const AdapterKernel &k, int n, int &count)
{
    for (const condensa_ctx::ClusterFit &f : ctx->cluster_fit)
        if (f.f == k.f && f.size == n) {
            count = f.count;
            return CONDENSA_OK;
        }
    const int rc = allow_smem(ctx, k);
    if (rc) return rc;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)n);
    cfg.blockDim = dim3((unsigned)k.threads);
    cfg.dynamicSmemBytes = (size_t)k.smem;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)n;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    count = 0;
    CU_TRY(ctx, cudaOccupancyMaxActiveClusters(&count, k.f, &cfg));
    if (count < 1) return fail(ctx, CONDENSA_ERR_INTERNAL, "no cluster of %d CTAs fits the device", n);
    ctx->cluster_fit.push_back({k.f, n, count});
    return CONDENSA_OK;
}

// How many CTAs share a tile of the row kernel (a cluster: columns of both sides), and how many clusters share its
// destination columns, each of them forming h again. Taken is what a simple account of the rounds makes least: a CTA's
// time goes with its columns, those of the destination counting twice, plus some fixed work (about 600 columns' worth);
// two CTAs on an SM take 1.2 times as long as one. Measured at 12 tiles of 1500 -> 33278 columns in fp32: cluster 8
// alone 106 us, the choice (7, 3) 73 us; at 131 tiles of 4096 -> 4096 in bf16: cluster 4 50 us, the choice (2, 1) 45 us.
int choose_shape(condensa_ctx *ctx, const AdapterKernel &k, long long tiles, long long ws, long long wd, int &cluster, int &splits)
{
    double best = 0.0;
    for (int c = 1; c <= AD_MAX_CLUSTER; ++c) {
        int fit = 0;
        const int rc = resident_clusters(ctx, k, c, fit);
        if (rc) return rc;
        for (int s = 1; s <= (wd ? AD_MAX_CLUSTER : 1); ++s) {
            const long long n = tiles * s, full = n / fit, rest = n % fit;
            const double w = (double)ws / c + 2.0 * (double)wd / (c * s), crowded = 1.2 * w + 600.0;
            double t = (double)full * crowded;
            if (rest) t += rest * c > ctx->num_sms ? crowded : w + 600.0;
            if ((c == 1 && s == 1) || t < 0.999 * best) {
                best = t;
                cluster = c;
                splits = s;
            }
        }
    }
    return CONDENSA_OK;
}

AdapterKernel row_kernel_of(int dtype, const RowShape &s)
{
    return dtype == CONDENSA_DTYPE_BF16 ? row_kernel<__nv_bfloat16>(s) : dtype == CONDENSA_DTYPE_FP16 ? row_kernel<__half>(s) : row_kernel<float>(s);
}

AdapterKernel wgrad_kernel_of(int dtype, int rank, int vec, int &strip)
{
    return dtype == CONDENSA_DTYPE_BF16 ? wgrad_kernel<__nv_bfloat16>(rank, vec, strip)
         : dtype == CONDENSA_DTYPE_FP16 ? wgrad_kernel<__half>(rank, vec, strip) : wgrad_kernel<float>(rank, vec, strip);
}

// ------------------------------------------------------------------ adapters laid out anew
constexpr size_t NONE = ~(size_t)0;
struct Packed {
    std::vector<size_t> a, b;           // byte offsets in the workspace, of used[i]; NONE: used as it is
    size_t bytes = 0;
    bool trans = false;
};

long long packed_ld(long long width, int e) { return (width * e + 15) / 16 * 16 / e; }

// `vec`: access width of the row kernel. It reads rows of A by 16 bytes (8 where vec is 8), rows of B by 8.
void plan_packing(const condensa_adapter_batch *b, const Rows &rows, bool trans, int vec, Packed &pk)
{
    const int e = type_bytes(b->dtype);
    pk.trans = trans;
    pk.a.assign(rows.used.size(), NONE);
    pk.b.assign(rows.used.size(), NONE);
    for (size_t i = 0; i < rows.used.size(); ++i) {
        const condensa_adapter &x = b->adapters[rows.used[i]];
        if (trans || widest(x.a, b->k * e) < (vec == 8 ? 8 : 16)) {
            pk.a[i] = pk.bytes;
            pk.bytes += align_up((size_t)((trans ? b->k * packed_ld(x.rank, e) : x.rank * packed_ld(b->k, e)) * e), 256);
        }
        if (trans || widest(x.b, (long long)x.rank * e) < 8) {
            pk.b[i] = pk.bytes;
            pk.bytes += align_up((size_t)((trans ? x.rank * packed_ld(b->n, e) : b->n * packed_ld(x.rank, e)) * e), 256);
        }
    }
}

int run_packing(condensa_ctx *ctx, const condensa_adapter_batch *b, const Rows &rows, const Packed &pk, char *ws, cudaStream_t stream)
{
    const int e = type_bytes(b->dtype);
    PackParams P;
    P.n = 0;
    long long blocks = 0;
    auto flush = [&]() -> int {
        if (!P.n) return CONDENSA_OK;
        const int pa_ = prof_begin(ctx, "k_adapter_pack", stream);
        if (e == 2) k_adapter_pack<u16><<<(unsigned)blocks, THREADS, 0, stream>>>(P);
        else k_adapter_pack<u32><<<(unsigned)blocks, THREADS, 0, stream>>>(P);
        LAUNCH_CHECK(ctx);
        prof_end(ctx, pa_, stream);
        P.n = 0;
        blocks = 0;
        return CONDENSA_OK;
    };
    for (size_t i = 0; i < rows.used.size(); ++i) {
        const condensa_adapter &x = b->adapters[rows.used[i]];
        for (int side = 0; side < 2; ++side) {
            const size_t at = side ? pk.b[i] : pk.a[i];
            if (at == NONE) continue;
            const long long r = side ? b->n : x.rank, w = side ? x.rank : b->k;
            // (a tile past the rows covers the padding of transposed rows)
            const long long ld = packed_ld(pk.trans ? r : w, e), T = AD_PACK_TILE;
            const long long tiles = ((pk.trans ? ld : r) + T - 1) / T * (((pk.trans ? w : ld) + T - 1) / T);
            if (P.n == AD_PACK_MAX || (P.n && blocks + tiles > 0x7FFFFFFFll)) {
                const int rc = flush();
                if (rc) return rc;
            }
            P.item[P.n++] = {side ? x.b : x.a, ws + at, r, w, (int)ld, pk.trans ? 1 : 0, (int)blocks, 0};
            blocks += tiles;
        }
    }
    return flush();
}

// ------------------------------------------------------------------ both directions of the row kernel
struct RowCall {
    const void *src;
    void *dst;
    float *h;
    long long ld_src, ld_dst, ld_h;
    bool trans;
    int vec;                // accesses that the rows of src and dst allow: 16, 8, or 0 for less
};

RowCall row_call(const void *src, void *dst, float *h, long long ld_src, long long ld_dst, long long ld_h, bool trans, int e)
{
    const int v = std::min(widest(src, ld_src * e), dst ? widest(dst, ld_dst * e) : 16);
    return {src, dst, h, ld_src, ld_dst, ld_h, trans, v >= 8 ? v : 0};
}

int run_rows(condensa_ctx *ctx, const condensa_adapter_batch *b, const Rows &rows, const Packed &pk, const char *pk_ws, const RowCall &c, cudaStream_t stream)
{
    const int e = type_bytes(b->dtype);
    // tiles of 64 rows where the adapters have that many; for a few rows each, 16 waste less and spread further
    const int tm = rows.live >= 48ll * (long long)rows.used.size() ? 64 : 16;
    long long all = 0;
    for (int n : rows.count) all += (n + tm - 1) / tm;
    const AdapterKernel kernel = row_kernel_of(b->dtype, {tm, rows.max_rank, c.vec});
    const long long ws = c.trans ? b->n : b->k, wd = c.dst ? (c.trans ? b->k : b->n) : 0;
    int cluster = 1, splits = 1;
    int rc = choose_shape(ctx, kernel, all, ws, wd, cluster, splits);
    if (rc) return rc;
    AdapterParams P;
    memset(&P, 0, offsetof(AdapterParams, blob));
    P.src = c.src; P.dst = c.dst; P.h = c.h;
    P.ld_src = c.ld_src; P.ld_dst = c.ld_dst; P.ld_h = c.ld_h;
    P.width_src = ws;
    P.width_dst = c.trans ? b->k : b->n;
    P.vec_src = widest(c.src, c.ld_src * e);
    P.vec_dst = c.dst ? widest(c.dst, c.ld_dst * e) : 16;
    P.splits = splits;
    P.scale_h = c.trans ? 1 : 0;
    Blob<AdapterEntry> blob;
    int tiles = 0;
    auto flush = [&]() -> int {
        P.n_entries = (int)blob.entries.size();
        blob.write(P.blob);
        rc = launch_cluster(ctx, kernel, dim3((unsigned)(tiles * cluster * P.splits)), dim3((unsigned)cluster), pk.bytes != 0, &P,
                                      c.trans ? "k_adapter_backward" : "k_adapter_forward", stream);
        blob.clear();
        tiles = 0;
        return rc;
    };
    for (size_t i = 0; i < rows.used.size(); ++i) {
        const condensa_adapter &ad = b->adapters[rows.used[i]];
        for (int run = rows.begin[i]; run < rows.end[i];) {
            // (an adapter is cut only where its runs fill a launch's parameters by themselves)
            if (!blob.entries.empty() && blob.room() < rows.end[i] - run && (rc = flush()) != 0) return rc;
            const int to = std::min(rows.end[i], run + blob.room());
            const bool pa = pk.a[i] != NONE, pb = pk.b[i] != NONE;
            const void *am = pa ? pk_ws + pk.a[i] : (const char *)ad.a, *bm = pb ? pk_ws + pk.b[i] : (const char *)ad.b;
            AdapterEntry en;
            memset(&en, 0, sizeof(en));
            if (c.trans) {
                en.shrink = bm; en.ld_s = (int)packed_ld(b->n, e);
                en.expand = am; en.ld_e = (int)packed_ld(ad.rank, e);
            } else {
                en.shrink = am; en.ld_s = (int)(pa ? packed_ld(b->k, e) : b->k);
                en.expand = bm; en.ld_e = (int)(pb ? packed_ld(ad.rank, e) : ad.rank);
            }
            en.scale = ad.scale;
            en.rank = (u16)ad.rank;
            en.tile0 = tiles;
            blob.add(en, rows, run, to);
            tiles += (blob.entries.back().n_rows + tm - 1) / tm;
            run = to;
        }
    }
    return blob.entries.empty() ? CONDENSA_OK : flush();
}

// ------------------------------------------------------------------ weight gradients
struct Wgrad {
    const void *x, *dy;
    const float *u, *h;
    long long ldx, lddy, ldu, ldh;
    bool accumulate;
    bool behind;                        // the row kernel goes ahead
};

int run_wgrad(condensa_ctx *ctx, const condensa_adapter_batch *b, const Rows &rows, const Wgrad &w, cudaStream_t stream)
{
    const int e = type_bytes(b->dtype);
    WgradParams P;
    memset(&P, 0, offsetof(WgradParams, blob));
    P.side[0] = {w.x, w.u, w.ldx, w.ldu, b->k, w.x ? widest(w.x, w.ldx * e) : 16, w.u ? widest(w.u, w.ldu * 4) : 16};
    P.side[1] = {w.dy, w.h, w.lddy, w.ldh, b->n, w.dy ? widest(w.dy, w.lddy * e) : 16, w.h ? widest(w.h, w.ldh * 4) : 16};
    const int v = std::min(P.side[0].vec_act, P.side[1].vec_act), vec = v >= 8 ? v : 0;
    Blob<WgEntry> blob;
    int rank = 1, most_tiles = 1;
    bool first = w.behind;
    auto flush = [&](bool accumulate) -> int {
        P.n_entries = (int)blob.entries.size();
        P.accumulate = accumulate ? 1 : 0;
        blob.write(P.blob);
        int strip;
        const AdapterKernel kernel = wgrad_kernel_of(b->dtype, rank, vec, strip);
        P.strips0 = (int)((b->k + strip - 1) / strip);
        const int strips = P.strips0 + (int)((b->n + strip - 1) / strip);
        // CTAs that share an adapter's rows: what a simple account makes least. A CTA's time is its tiles and about four
        // tiles' worth of fixed work; two on an SM take 1.3 times as long as one; CTAs past the first round follow as places
        // free up. Measured on 4 adapters of 2048 rows, 32 strips: 1: 79, 2: 53, 3: 49, 4: 49, 8: 63 us; on 6 of 430 rows,
        // 30 strips: 1: 53, 2: 45, 3: 50, 4: 63 us.
        int cluster = 1;
        double best = 0.0;
        for (int n = 1; n <= std::min(AD_MAX_CLUSTER, most_tiles); ++n) {
            const long long ctas = (long long)strips * P.n_entries * n;
            const double rounds = std::max(1.0, (double)ctas / (double)(ctx->num_sms * kernel.per_sm / n * n));
            const double t = rounds * ((double)((most_tiles + n - 1) / n) + 4.0) * (ctas > ctx->num_sms ? 1.3 : 1.0);
            if (n == 1 || t < 0.999 * best) {
                best = t;
                cluster = n;
            }
        }
        const int rc = launch_cluster(ctx, kernel, dim3((unsigned)strips, (unsigned)(P.n_entries * cluster)), dim3(1, (unsigned)cluster), first, &P,
                                      "k_adapter_wgrad", stream);
        blob.clear();
        rank = most_tiles = 1;
        first = false;
        return rc;
    };
    size_t u = 0;
    for (int a = 0; a < b->n_adapters; ++a) {
        const condensa_adapter &ad = b->adapters[a];
        const bool live = u < rows.used.size() && rows.used[u] == a;
        const size_t i = u;
        if (live) ++u;
        if ((!ad.grad_a && !ad.grad_b) || (!live && w.accumulate)) continue;
        int run = live ? rows.begin[i] : 0;
        const int end = live ? rows.end[i] : 0;
        bool more = false;
        do {            // once, but where an adapter's runs fill a launch's parameters by themselves: the rest is added
            if (!blob.entries.empty() && (more || blob.room() < end - run)) {
                const int rc = flush(w.accumulate);
                if (rc) return rc;
            }
            const int to = std::min(end, run + blob.room());
            WgEntry en;
            memset(&en, 0, sizeof(en));
            en.out[0] = ad.grad_a;
            en.out[1] = ad.grad_b;
            en.scale = ad.scale;
            en.rank = ad.rank;
            blob.add(en, rows, run, to);
            rank = std::max(rank, (int)ad.rank);
            most_tiles = std::max(most_tiles, (blob.entries.back().n_rows + AD_WG_ROWS - 1) / AD_WG_ROWS);
            run = to;
            if (more || run < end) {
                const int rc = flush(more || w.accumulate);
                if (rc) return rc;
                more = true;
            }
        } while (run < end);
    }
    return blob.entries.empty() ? CONDENSA_OK : flush(w.accumulate);
}

// ------------------------------------------------------------------ calls
struct Ranges {
    std::vector<Interval> iv;
    std::vector<RowRange> rows;
    void add(const void *p, long long bytes, bool out)
    {
        if (p && bytes > 0) iv.push_back({(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, out});
    }
    bool clash() { return rows_clash(iv, rows); }
};

// A matrix of `rows` x `width` values: checked, and its range noted.
int take_rows(condensa_ctx *ctx, const char *name, const void *p, long long ld, long long rows, long long width, int e, bool out, Ranges &r)
{
    if (rows == 0) return CONDENSA_OK;
    if (!p) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "%s is NULL", name);
    if ((uintptr_t)p % e) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "%s is not aligned to its type", name);
    if (ld < width) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "%s: rows of %lld values lie %lld apart", name, width, ld);
    if (width == 0) return CONDENSA_OK;          // (h where no row has an adapter)
    if (ld > (1ll << 40) || rows - 1 > (1ll << 56) / ld) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "%s: %lld rows %lld apart leave the address space", name, rows, ld);
    r.rows.push_back({(uintptr_t)p, (uintptr_t)(width * e), (uintptr_t)(ld * e), (uintptr_t)rows, out});
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
    if (r.clash()) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "an output buffer overlaps another buffer of the call");
    if (rows.live == 0) return CONDENSA_OK;
    CU_TRY(ctx, cudaSetDevice(ctx->device));
    const RowCall call = row_call(x, y, h, ldx, ldy, ldh, false, e);
    Packed pk;
    plan_packing(b, rows, false, call.vec, pk);
    char *ws = nullptr;
    OpWorkspaceUse use;
    if (pk.bytes) {
        if ((rc = op_workspace(ctx, 256 + pk.bytes, stream, use)) != 0) return rc;
        ws = ctx->op.p + 256;
        if ((rc = run_packing(ctx, b, rows, pk, ws, stream)) != 0) return rc;
    }
    if ((rc = run_rows(ctx, b, rows, pk, ws, call, stream)) != 0) return rc;
    return op_workspace_done(ctx, use);
}

int backward(condensa_ctx *ctx, const condensa_adapter_batch *b, const void *x, long long ldx, const void *dy, long long lddy, const float *h,
             long long ldh, void *dx, long long lddx, int accumulate, cudaStream_t stream)
{
    Rows rows;
    int rc = read_batch(ctx, b, rows);
    if (rc) return rc;
    const int e = type_bytes(b->dtype);
    bool need_a = false, need_b = false;       // a grad_a, a grad_b of an adapter with rows
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
        r.add(ad.grad_a, (long long)ad.rank * b->k * 4, true);
        r.add(ad.grad_b, (long long)ad.rank * b->n * 4, true);
    }
    if (r.clash()) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "an output buffer overlaps another buffer of the call");
    CU_TRY(ctx, cudaSetDevice(ctx->device));
    const bool row_kernel = rows.live && (dx || need_a);
    Packed pk;
    if (row_kernel) plan_packing(b, rows, true, 16, pk);
    const long long ldu = (rows.max_rank + 3) / 4 * 4;
    const size_t u_bytes = need_a ? align_up(sizeof(float) * (size_t)(rows.total * ldu), 256) : 0;
    float *u_ws = nullptr;
    char *pk_ws = nullptr;
    OpWorkspaceUse use;
    if (u_bytes + pk.bytes) {
        if ((rc = op_workspace(ctx, 256 + u_bytes + pk.bytes, stream, use)) != 0) return rc;
        u_ws = need_a ? (float *)(ctx->op.p + 256) : nullptr;
        pk_ws = ctx->op.p + 256 + u_bytes;
    }
    if (pk.bytes && (rc = run_packing(ctx, b, rows, pk, pk_ws, stream)) != 0) return rc;
    if (row_kernel && (rc = run_rows(ctx, b, rows, pk, pk_ws, row_call(dy, dx, u_ws, lddy, lddx, ldu, true, e), stream)) != 0) return rc;
    if ((rc = run_wgrad(ctx, b, rows, {x, dy, u_ws, h, ldx, lddy, ldu, ldh, accumulate != 0, row_kernel}, stream)) != 0) return rc;
    return op_workspace_done(ctx, use);
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
