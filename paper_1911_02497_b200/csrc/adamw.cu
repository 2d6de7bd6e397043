// Host side of the AdamW step and the gradient norm: argument checks, descriptors, launches.
#include <cmath>
#include <new>

#include "adamw.cuh"
#include "ctx.cuh"

using namespace cs;

static_assert(CONDENSA_DTYPE_FP32 == GT_F32 && CONDENSA_DTYPE_FP16 == GT_F16 && CONDENSA_DTYPE_BF16 == GT_BF16, "type codes");
static_assert(CONDENSA_STATE_BLOCK == LIST_CHUNK, "block of the 8-bit states");

namespace {

constexpr int GROUP = WARPS * LIST_CHUNK;       // elements of one step of a CTA

struct ListCheck {
    int grad_dtype;
    bool step;              // false: only what the norm reads
    bool eight;
    int copy_dtype;
};

// Checks the list and fills `d`; `pen` is set when a tensor has a theta.
int check_list(condensa_ctx *ctx, const condensa_adamw_tensor *ts, int T, const ListCheck &c, std::vector<ListDesc> &d, bool &pen)
{
    std::vector<Interval> iv;
    iv.reserve((size_t)T * 9);
    d.resize((size_t)T);
    pen = false;
    const size_t gsize = c.grad_dtype == CONDENSA_DTYPE_FP32 ? 4 : 2, ssize = c.eight ? 1 : 4;
    for (int t = 0; t < T; ++t) {
        const condensa_adamw_tensor &x = ts[t];
        ListDesc &o = d[t];
        memset(&o, 0, sizeof(o));
        if (x.numel < 0) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "tensor %d: numel < 0", t);
        if (x.numel == 0) continue;
        if (x.numel > (1ll << 40)) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "tensor %d: more than 2^40 elements", t);
        const bool has_th = x.theta != nullptr;
        if (!x.grad) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "tensor %d: grad is NULL", t);
        if ((c.step || has_th) && !x.w) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "tensor %d: w is NULL", t);
        if (c.step && (!x.m || !x.v)) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "tensor %d: a moment is NULL", t);
        if (c.step && c.eight && (!x.m_scale || !x.v_scale)) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "tensor %d: a scale of the 8-bit states is NULL", t);
        if (c.step && x.w_h && c.copy_dtype != CONDENSA_DTYPE_FP16 && c.copy_dtype != CONDENSA_DTYPE_BF16)
            return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "w_h_dtype must be CONDENSA_DTYPE_FP16 or CONDENSA_DTYPE_BF16");
        const size_t n = (size_t)x.numel, blocks = (n + LIST_CHUNK - 1) / LIST_CHUNK;
        bool vec = true, natural = true;
        // bytes per element, bytes of a quad access (0: never accessed in quads), written
        auto take = [&](const void *p, size_t bytes, size_t size, size_t quad, bool out) {
            if (!p) return;
            if ((uintptr_t)p % size) natural = false;
            if (quad && (uintptr_t)p % quad) vec = false;
            iv.push_back({(uintptr_t)p, (uintptr_t)p + bytes, out});
        };
        take(x.grad, n * gsize, gsize, 4 * gsize, false);
        if (c.step || has_th) take(x.w, 4 * n, 4, 16, c.step);
        if (has_th) {
            take(x.theta, 4 * n, 4, 16, false);
            take(x.lambda, 4 * n, 4, 16, false);
            pen = true;
        }
        if (c.step) {
            take(x.m, n * ssize, ssize, 4 * ssize, true);
            take(x.v, n * ssize, ssize, 4 * ssize, true);
            if (c.eight) {
                take(x.m_scale, 4 * blocks, 4, 0, true);
                take(x.v_scale, 4 * blocks, 4, 0, true);
            }
            take(x.w_h, 2 * n, 2, 8, true);
        }
        if (!natural) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "tensor %d: a pointer is not aligned to its type", t);
        o.w = x.w;
        o.theta = x.theta;
        o.lam = has_th ? x.lambda : nullptr;
        o.grad = x.grad;
        if (c.step) {
            o.m = x.m;
            o.v = x.v;
            o.m_scale = c.eight ? x.m_scale : nullptr;
            o.v_scale = c.eight ? x.v_scale : nullptr;
            o.w_h = x.w_h;
        }
        o.numel = x.numel;
        o.vec_ok = vec ? 1u : 0u;
    }
    if (c.step && ranges_clash(iv)) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "an in/out buffer overlaps another buffer of the call");
    return CONDENSA_OK;
}

// Work items of tensors [t0, t0 + T): `chunks` groups of a CTA each, so many that the grid still has
// several items per CTA (a descriptor search per item), but a short list is spread over all SMs.
int set_items(condensa_ctx *ctx, ListDesc *d, int T, int grid_max, ListScalars &s)
{
    long long groups = 0;
    for (int t = 0; t < T; ++t) groups += (d[t].numel + GROUP - 1) / GROUP;
    s.chunks = groups >= 16ll * grid_max ? 4 : groups >= 6ll * grid_max ? 2 : 1;
    long long items = 0;
    for (int t = 0; t < T; ++t) {
        d[t].item0 = (u32)items;
        items += ((d[t].numel + GROUP - 1) / GROUP + s.chunks - 1) / s.chunks;
    }
    if (items > 0x7FFFFFFFll) return fail(ctx, CONDENSA_ERR_TOO_LARGE, "the list is too long for one launch");
    s.n_items = (u32)items;
    s.T = T;
    return CONDENSA_OK;
}

template <int CAP, int GT, int STATES, bool PEN>
void launch_adamw(const ListScalars &s, const ListDesc *d, int grid, cudaStream_t stream)
{
    ListParams<CAP> P;
    P.s = s;
    memcpy(P.d, d, sizeof(ListDesc) * (size_t)s.T);
    k_adamw<CAP, GT, STATES, PEN><<<grid, THREADS, 0, stream>>>(P);
}

template <int CAP, int GT>
void launch_adamw_of(int states, bool pen, const ListScalars &s, const ListDesc *d, int grid, cudaStream_t stream)
{
    if (states == ST_8_NEAREST) pen ? launch_adamw<CAP, GT, ST_8_NEAREST, true>(s, d, grid, stream) : launch_adamw<CAP, GT, ST_8_NEAREST, false>(s, d, grid, stream);
    else if (states == ST_8_STOCHASTIC) pen ? launch_adamw<CAP, GT, ST_8_STOCHASTIC, true>(s, d, grid, stream) : launch_adamw<CAP, GT, ST_8_STOCHASTIC, false>(s, d, grid, stream);
    else pen ? launch_adamw<CAP, GT, ST_32, true>(s, d, grid, stream) : launch_adamw<CAP, GT, ST_32, false>(s, d, grid, stream);
}

template <int CAP>
void launch_adamw_cap(int gt, int states, bool pen, const ListScalars &s, const ListDesc *d, int grid, cudaStream_t stream)
{
    if (gt == GT_F32) launch_adamw_of<CAP, GT_F32>(states, pen, s, d, grid, stream);
    else if (gt == GT_F16) launch_adamw_of<CAP, GT_F16>(states, pen, s, d, grid, stream);
    else launch_adamw_of<CAP, GT_BF16>(states, pen, s, d, grid, stream);
}

template <int CAP, int GT, bool PEN>
void launch_norm(const ListScalars &s, const ListDesc *d, const NormOut &N, int grid, cudaStream_t stream)
{
    ListParams<CAP> P;
    P.s = s;
    memcpy(P.d, d, sizeof(ListDesc) * (size_t)s.T);
    k_grad_norm<CAP, GT, PEN><<<grid, THREADS, 0, stream>>>(P, N);
}

template <int CAP>
void launch_norm_cap(int gt, bool pen, const ListScalars &s, const ListDesc *d, const NormOut &N, int grid, cudaStream_t stream)
{
    if (gt == GT_F32) pen ? launch_norm<CAP, GT_F32, true>(s, d, N, grid, stream) : launch_norm<CAP, GT_F32, false>(s, d, N, grid, stream);
    else if (gt == GT_F16) pen ? launch_norm<CAP, GT_F16, true>(s, d, N, grid, stream) : launch_norm<CAP, GT_F16, false>(s, d, N, grid, stream);
    else pen ? launch_norm<CAP, GT_BF16, true>(s, d, N, grid, stream) : launch_norm<CAP, GT_BF16, false>(s, d, N, grid, stream);
}

bool known_grad_type(int t) { return t == CONDENSA_DTYPE_FP32 || t == CONDENSA_DTYPE_FP16 || t == CONDENSA_DTYPE_BF16; }

int adamw(condensa_ctx *ctx, const condensa_adamw_tensor *ts, int T, float mu, const condensa_adamw *opt,
          const condensa_clip *clip, cudaStream_t stream)
{
    if (!ts || T <= 0 || T > (1 << 20) || !opt) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "tensor list or optimizer is NULL or empty");
    if (!known_grad_type(opt->grad_dtype)) return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "grad_dtype must be CONDENSA_DTYPE_FP32, _FP16 or _BF16");
    if (opt->state_dtype != CONDENSA_DTYPE_FP32 && opt->state_dtype != CONDENSA_DTYPE_FP8_E4M3)
        return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "state_dtype must be CONDENSA_DTYPE_FP32 or CONDENSA_DTYPE_FP8_E4M3");
    if (!std::isfinite(opt->lr) || !std::isfinite(opt->weight_decay) || !std::isfinite(opt->grad_scale))
        return fail(ctx, CONDENSA_ERR_INVALID_ARG, "optimizer parameters must be finite");
    if (!(opt->beta1 >= 0.0f && opt->beta1 < 1.0f) || !(opt->beta2 >= 0.0f && opt->beta2 < 1.0f) || opt->step < 1 || !(opt->eps >= 0.0f) ||
        !std::isfinite(opt->eps))
        return fail(ctx, CONDENSA_ERR_INVALID_ARG, "AdamW needs 0 <= beta < 1, eps >= 0 and step >= 1");
    if ((uintptr_t)clip % 4) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "clip is not 4-byte aligned");
    std::vector<ListDesc> d;
    bool pen = false;
    const bool eight = opt->state_dtype == CONDENSA_DTYPE_FP8_E4M3;
    int rc = check_list(ctx, ts, T, {opt->grad_dtype, true, eight, opt->w_h_dtype}, d, pen);
    if (rc) return rc;
    if (pen && (!(mu >= 0.0f) || !std::isfinite(mu))) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "mu must be finite and >= 0");
    CU_TRY(ctx, cudaSetDevice(ctx->device));
    ListScalars s;
    memset(&s, 0, sizeof(s));
    s.mu = mu;
    s.grad_scale = opt->grad_scale;
    s.beta1 = opt->beta1;
    s.beta2 = opt->beta2;
    s.c1 = 1.0f - opt->beta1;
    s.c2 = 1.0f - opt->beta2;
    s.decay = (float)(1.0 - (double)opt->lr * (double)opt->weight_decay);
    s.step_size = (float)((double)opt->lr / (1.0 - std::pow((double)opt->beta1, (double)opt->step)));
    s.root_corr = (float)(1.0 / std::sqrt(1.0 - std::pow((double)opt->beta2, (double)opt->step)));
    s.eps = opt->eps;
    s.clip = (const float *)clip;
    s.copy_type = opt->w_h_dtype;
    s.key = mix64(mix64(opt->state_seed) ^ (u64)opt->step);
    const int states = !eight ? ST_32 : opt->state_seed ? ST_8_STOCHASTIC : ST_8_NEAREST;
    const int per_sm = adamw_ctas(states, pen), grid_max = ctx->num_sms * per_sm;
    for (int t0 = 0; t0 < T; t0 += LIST_LARGE) {
        const int n = std::min(T - t0, LIST_LARGE);
        if ((rc = set_items(ctx, d.data() + t0, n, grid_max, s)) != 0) return rc;
        if (s.n_items == 0) continue;
        s.t0 = t0;
        const int grid = stream_grid(ctx, s.n_items, per_sm);
        const int pa_ = prof_begin(ctx, eight ? "k_adamw_8" : "k_adamw_32", stream);
        if (n <= LIST_SMALL) launch_adamw_cap<LIST_SMALL>(opt->grad_dtype, states, pen, s, d.data() + t0, grid, stream);
        else launch_adamw_cap<LIST_LARGE>(opt->grad_dtype, states, pen, s, d.data() + t0, grid, stream);
        LAUNCH_CHECK(ctx);
        prof_end(ctx, pa_, stream);
    }
    return CONDENSA_OK;
}

int grad_norm(condensa_ctx *ctx, const condensa_adamw_tensor *ts, int T, float mu, int grad_dtype, float grad_scale,
              float max_norm, condensa_clip *clip, float *norms, cudaStream_t stream)
{
    if (!ts || T <= 0 || T > (1 << 20)) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "tensor list is empty or NULL");
    if (!known_grad_type(grad_dtype)) return fail(ctx, CONDENSA_ERR_UNSUPPORTED, "grad_dtype must be CONDENSA_DTYPE_FP32, _FP16 or _BF16");
    if (!std::isfinite(grad_scale) || std::isnan(max_norm)) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "grad_scale must be finite and max_norm a number");
    if (!clip || (uintptr_t)clip % 4 || (uintptr_t)norms % 4) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "clip is NULL, or clip or norms misaligned");
    std::vector<ListDesc> d;
    bool pen = false;
    int rc = check_list(ctx, ts, T, {grad_dtype, false, false, 0}, d, pen);
    if (rc) return rc;
    if (pen && (!(mu >= 0.0f) || !std::isfinite(mu))) return fail(ctx, CONDENSA_ERR_INVALID_ARG, "mu must be finite and >= 0");
    CU_TRY(ctx, cudaSetDevice(ctx->device));
    const int grid_max = std::min(ctx->num_sms * 4, NORM_GRID_MAX);
    const size_t slots = (size_t)grid_max + LIST_LARGE;
    OpWorkspaceUse use;
    rc = op_workspace(ctx, 256 + sizeof(double) * (slots + (size_t)T), stream, use);
    if (rc) return rc;
    NormOut N;
    N.done = (u32 *)ctx->op.p;
    N.slot = (double *)(ctx->op.p + 256);
    N.square = N.slot + slots;
    N.norms = norms;
    N.clip = (float *)clip;
    N.T_all = T;
    N.max_norm = max_norm;
    ListScalars s;
    memset(&s, 0, sizeof(s));
    s.mu = mu;
    s.grad_scale = grad_scale;
    for (int t0 = 0; t0 < T; t0 += LIST_LARGE) {
        const int n = std::min(T - t0, LIST_LARGE);
        if ((rc = set_items(ctx, d.data() + t0, n, grid_max, s)) != 0) return rc;
        N.t0 = t0;
        N.last = t0 + n == T;
        const int grid = std::max(1, std::min(grid_max, (int)s.n_items));
        const int pa_ = prof_begin(ctx, "k_grad_norm", stream);
        if (n <= LIST_SMALL) launch_norm_cap<LIST_SMALL>(grad_dtype, pen, s, d.data() + t0, N, grid, stream);
        else launch_norm_cap<LIST_LARGE>(grad_dtype, pen, s, d.data() + t0, N, grid, stream);
        LAUNCH_CHECK(ctx);
        prof_end(ctx, pa_, stream);
    }
    return op_workspace_done(ctx, use);
}

}  // namespace

extern "C" {

int condensa_lstep_adamw(condensa_ctx *ctx, const condensa_adamw_tensor *tensors, int T, float mu, const condensa_adamw *opt,
                         const condensa_clip *clip, void *stream)
{
    if (!ctx) return CONDENSA_ERR_INVALID_ARG;
    try {
        return adamw(ctx, tensors, T, mu, opt, clip, (cudaStream_t)stream);
    } catch (const std::bad_alloc &) {
        return fail(ctx, CONDENSA_ERR_WORKSPACE, "out of host memory");
    }
}

int condensa_grad_norm(condensa_ctx *ctx, const condensa_adamw_tensor *tensors, int T, float mu, int grad_dtype, float grad_scale,
                       float max_norm, condensa_clip *clip, float *norms, void *stream)
{
    if (!ctx) return CONDENSA_ERR_INVALID_ARG;
    try {
        return grad_norm(ctx, tensors, T, mu, grad_dtype, grad_scale, max_norm, clip, norms, (cudaStream_t)stream);
    } catch (const std::bad_alloc &) {
        return fail(ctx, CONDENSA_ERR_WORKSPACE, "out of host memory");
    }
}

}  // extern "C"
