// C ABI of the block operators (declared in include/mosa.h): argument checks, workspace
// and dispatch of the residual step, dropout and the log probabilities.
#include <cmath>

#include "args.h"
#include "block.h"

namespace mosa {
namespace blk {
namespace {

constexpr int kMaxWidth = 8192;   // of the residual step's rows

mosa_status check_rows(int B, int T, int n) {
    if (B <= 0 || T <= 0 || n <= 0) return MOSA_ERR_INVALID_ARG;
    return (long long)B * T < (1LL << 31) ? MOSA_OK : MOSA_ERR_UNSUPPORTED;
}

bool dtype_ok(int t) { return t == MOSA_F32 || t == MOSA_BF16; }
bool flag_ok(int v) { return v == 0 || v == 1; }

// An optional pointer is at a multiple of its element's size.
bool place_ok(const void *p, int dtype) { return aligned(p, dtype); }
bool place8_ok(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 7) == 0; }

mosa_status check_drop(double p, int site, const int64_t *rng, Drop *d) {
    if (!(p >= 0.0) || !(p <= 1.0)) return MOSA_ERR_INVALID_ARG;
    if (p > 0.0 && (rng == nullptr || !place8_ok(rng))) return MOSA_ERR_INVALID_ARG;
    *d = Drop{p > 0.0 ? rng : nullptr, site, (uint64_t)std::nearbyint(p * 4294967296.0),
              p < 1.0 ? (float)(1.0 / (1.0 - p)) : 0.f};
    return MOSA_OK;
}

// Sizes, flags and strides (no pointers).
mosa_status check_residual(const mosa_residual_shape *s, bool backward, Residual *r, Str *str) {
    if (s == nullptr) return MOSA_ERR_INVALID_ARG;
    mosa_status st = check_rows(s->B, s->T, s->d);
    if (st != MOSA_OK) return st;
    if (!dtype_ok(s->dtype) || !dtype_ok(s->x_dtype) || !dtype_ok(s->y_dtype)) return MOSA_ERR_INVALID_ARG;
    if (!flag_ok(s->post_norm) || !flag_ok(s->pre_norm) || !flag_ok(s->sigmoid)) return MOSA_ERR_INVALID_ARG;
    if (s->gate < MOSA_GATE_NONE || s->gate > MOSA_GATE_TOKEN) return MOSA_ERR_INVALID_ARG;
    if (!std::isfinite(s->scale) || !(s->eps >= 0.f) || std::isinf(s->eps)) return MOSA_ERR_INVALID_ARG;
    if (!(s->dropout >= 0.0) || !(s->dropout <= 1.0)) return MOSA_ERR_INVALID_ARG;
    if (s->d > kMaxWidth) return MOSA_ERR_UNSUPPORTED;
    *r = Residual{};
    r->B = s->B;
    r->T = s->T;
    r->d = s->d;
    r->post = s->post_norm;
    r->pre = s->pre_norm;
    r->gate = s->gate;
    r->sigmoid = s->sigmoid;
    r->storage_wide = s->dtype == MOSA_F32;
    r->scale = s->scale;
    r->eps = s->eps;
    const bool token = s->gate == MOSA_GATE_TOKEN;
    const mosa_strides *in[10] = {&s->x, &s->y, &s->g, &s->xo, &s->h, &s->dxo, &s->dh, &s->dx, &s->dy, &s->dg};
    for (int i = 0; i < 10; ++i) {
        if (i == 2 && !token) continue;
        if (i == 4 && !s->pre_norm) continue;
        if (i >= 5 && !backward) break;
        if (i == 9 && !token) continue;
        if (i == 6 && !s->pre_norm) continue;
        if ((i == 3 || i == 4) && backward) continue;
        const mosa_strides v = {in[i]->b, in[i]->t, 0};
        if (!strides(v, s->B, s->T, 1, &str[i])) return MOSA_ERR_INVALID_ARG;
        if ((i == 3 || i == 4 || i >= 7) && !output(str[i], s->B, s->T, 1, s->d)) return MOSA_ERR_INVALID_ARG;
    }
    if (backward && s->pre_norm && !dtype_ok(s->dh_dtype)) return MOSA_ERR_INVALID_ARG;
    return MOSA_OK;
}

Vec vec_of(const void *p, int dtype) { return Vec{p, dtype == MOSA_F32, (uintptr_t)p % 16 == 0}; }

// Inputs that both directions share.
mosa_status take_inputs(const mosa_residual_shape *s, const void *x, const void *y, const void *gate,
                        const void *gamma_post, const void *gamma_pre, const int64_t *rng,
                        const Str *str, Residual *r) {
    if (check_ptrs(s->x_dtype, {x}) != MOSA_OK || check_ptrs(s->y_dtype, {y}) != MOSA_OK)
        return MOSA_ERR_INVALID_ARG;
    if (s->gate != MOSA_GATE_NONE && check_ptrs(s->dtype, {gate}) != MOSA_OK) return MOSA_ERR_INVALID_ARG;
    if (!place_ok(gamma_post, s->dtype) || !place_ok(gamma_pre, s->dtype)) return MOSA_ERR_INVALID_ARG;
    mosa_status st = check_drop(s->dropout, s->site, rng, &r->drop);
    if (st != MOSA_OK) return st;
    r->x = rows_of(x, str[0], s->x_dtype);
    r->y = rows_of(y, str[1], s->y_dtype);
    if (s->gate == MOSA_GATE_TOKEN) r->g = rows_of(gate, str[2], s->dtype);
    if (s->gate == MOSA_GATE_CHANNEL) r->gch = vec_of(gate, s->dtype);
    r->gpost = vec_of(s->post_norm ? gamma_post : nullptr, s->dtype);
    r->gpre = vec_of(s->pre_norm ? gamma_pre : nullptr, s->dtype);
    return MOSA_OK;
}

mosa_status check_logprob(const mosa_logprob_shape *s, bool backward, LogProb *l, Str *z, Str *dz) {
    if (s == nullptr) return MOSA_ERR_INVALID_ARG;
    mosa_status st = check_rows(s->B, s->T, s->V);
    if (st != MOSA_OK) return st;
    if (!dtype_ok(s->dtype) || !flag_ok(s->target64) || !flag_ok(s->stats)) return MOSA_ERR_INVALID_ARG;
    if (s->top < 0 || s->top > s->V) return MOSA_ERR_INVALID_ARG;
    if (!(s->scale > 0.f) || std::isinf(s->scale)) return MOSA_ERR_INVALID_ARG;
    if (s->top > 32 || s->scale < 1.f / 1048576 || s->scale > 1048576.f) return MOSA_ERR_UNSUPPORTED;
    if (s->V >= 2147483647 - 65536) return MOSA_ERR_UNSUPPORTED;
    *l = LogProb{};
    l->B = s->B;
    l->T = s->T;
    l->V = s->V;
    l->target64 = s->target64;
    l->z.wide = l->dz.wide = s->dtype == MOSA_F32;
    l->top = s->top;
    l->stats = s->stats;
    l->scale = s->scale;
    const mosa_strides a = {s->z.b, s->z.t, 0}, b = {s->dz.b, s->dz.t, 0};
    if (!strides(a, s->B, s->T, 1, z)) return MOSA_ERR_INVALID_ARG;
    if (backward && (!strides(b, s->B, s->T, 1, dz) || !output(*dz, s->B, s->T, 1, s->V)))
        return MOSA_ERR_INVALID_ARG;
    return MOSA_OK;
}

bool targets_ok(const void *p, int target64) { return target64 ? place8_ok(p) : place_ok(p, MOSA_F32); }

bool floats_ok(std::initializer_list<const void *> ps) {
    for (const void *p : ps)
        if (!place_ok(p, MOSA_F32)) return false;
    return true;
}

mosa_status of(cudaError_t e) { return e == cudaSuccess ? MOSA_OK : MOSA_ERR_CUDA; }

}  // namespace
}  // namespace blk
}  // namespace mosa

using namespace mosa;
using namespace mosa::blk;

extern "C" {

mosa_status mosa_residual_forward(const mosa_residual_shape *shape, const void *x, const void *y,
                                  const void *gate, const void *gamma_post, const void *gamma_pre,
                                  const int64_t *rng, void *x_out, void *h, float *stats,
                                  void *stream) {
    Residual r;
    Str str[10];
    mosa_status st = check_residual(shape, false, &r, str);
    if (st != MOSA_OK) return st;
    if ((st = take_inputs(shape, x, y, gate, gamma_post, gamma_pre, rng, str, &r)) != MOSA_OK) return st;
    if (check_ptrs(shape->x_dtype, {x_out}) != MOSA_OK) return MOSA_ERR_INVALID_ARG;
    if (shape->pre_norm && check_ptrs(shape->dtype, {h}) != MOSA_OK) return MOSA_ERR_INVALID_ARG;
    if (!place_ok(stats, MOSA_F32)) return MOSA_ERR_INVALID_ARG;
    r.xo = rows_of(x_out, str[3], shape->x_dtype);
    if (shape->pre_norm) r.h = rows_of(h, str[4], shape->dtype);
    r.stats = stats;
    return of(launch_residual(r, (cudaStream_t)stream));
}

size_t mosa_residual_workspace_bytes(const mosa_residual_shape *shape) {
    Residual r;
    Str str[10];
    return check_residual(shape, true, &r, str) == MOSA_OK ? residual_workspace(r) : 0;
}

mosa_status mosa_residual_backward(const mosa_residual_shape *shape, const void *x, const void *y,
                                   const void *gate, const void *gamma_post,
                                   const void *gamma_pre, const int64_t *rng, const float *stats,
                                   const void *dx_out, const void *dh, void *dx, void *dy,
                                   void *dgate, float *dgamma_post, float *dgamma_pre,
                                   void *workspace, size_t workspace_bytes, void *stream) {
    Residual r;
    Str str[10];
    mosa_status st = check_residual(shape, true, &r, str);
    if (st != MOSA_OK) return st;
    if ((st = take_inputs(shape, x, y, gate, gamma_post, gamma_pre, rng, str, &r)) != MOSA_OK) return st;
    if (check_ptrs(MOSA_F32, {stats}) != MOSA_OK || check_ptrs(shape->x_dtype, {dx}) != MOSA_OK ||
        check_ptrs(shape->dtype, {dy}) != MOSA_OK)
        return MOSA_ERR_INVALID_ARG;
    const bool token = shape->gate == MOSA_GATE_TOKEN;
    if (!place_ok(dx_out, shape->x_dtype) || (shape->pre_norm && !place_ok(dh, shape->dh_dtype)) ||
        !place_ok(dgate, token ? shape->dtype : MOSA_F32) || !floats_ok({dgamma_post, dgamma_pre}))
        return MOSA_ERR_INVALID_ARG;
    if ((st = check_space(workspace, workspace_bytes, residual_workspace(r))) != MOSA_OK) return st;
    r.stats = const_cast<float *>(stats);
    if (shape->dropout >= 1.0) {   // nothing of y counts, nor of its norm, whatever they are
        r.post = 0;
        r.gpost = vec_of(nullptr, shape->dtype);
    }
    if (dx_out != nullptr) r.dxo = rows_of(dx_out, str[5], shape->x_dtype);
    if (shape->pre_norm && dh != nullptr) r.dh = rows_of(dh, str[6], shape->dh_dtype);
    r.dx = rows_of(dx, str[7], shape->x_dtype);
    r.dy = rows_of(dy, str[8], shape->dtype);
    if (token && dgate != nullptr) r.dg = rows_of(dgate, str[9], shape->dtype);
    if (shape->gate == MOSA_GATE_CHANNEL) r.dgate = static_cast<float *>(dgate);
    r.dgpost = dgamma_post;
    r.dgpre = dgamma_pre;
    return of(launch_residual_bwd(r, static_cast<float *>(workspace), (cudaStream_t)stream));
}

mosa_status mosa_dropout(const mosa_dropout_shape *shape, const void *x, const int64_t *rng, void *y,
                         void *stream) {
    if (shape == nullptr) return MOSA_ERR_INVALID_ARG;
    mosa_status st = check_rows(shape->B, shape->T, shape->d);
    if (st != MOSA_OK) return st;
    if (!dtype_ok(shape->dtype)) return MOSA_ERR_INVALID_ARG;
    // (runs of 256 columns are counted in 31 bits: a tensor that needs more has a terabyte)
    if ((long long)shape->B * shape->T * (shape->d / 256LL + 1) >= 1LL << 31 || shape->d >= 2147483647 - 65536)
        return MOSA_ERR_UNSUPPORTED;
    Drop d;
    if ((st = check_drop(shape->dropout, shape->site, rng, &d)) != MOSA_OK) return st;
    Str xs, ys;
    const mosa_strides a = {shape->x.b, shape->x.t, 0}, b = {shape->y.b, shape->y.t, 0};
    if (!strides(a, shape->B, shape->T, 1, &xs) || !strides(b, shape->B, shape->T, 1, &ys) ||
        !output(ys, shape->B, shape->T, 1, shape->d))
        return MOSA_ERR_INVALID_ARG;
    if ((st = check_ptrs(shape->dtype, {x, y})) != MOSA_OK) return st;
    return of(launch_dropout(shape->B, shape->T, shape->d, rows_of(x, xs, shape->dtype),
                             rows_of(y, ys, shape->dtype), d, (cudaStream_t)stream));
}

size_t mosa_token_logprobs_workspace_bytes(const mosa_logprob_shape *shape) {
    LogProb l;
    Str z, dz;
    return check_logprob(shape, false, &l, &z, &dz) == MOSA_OK ? logprob_workspace(l) : 0;
}

mosa_status mosa_token_logprobs(const mosa_logprob_shape *shape, const void *logits,
                                const void *targets, float *logp, float *entropy, float *lse,
                                int32_t *top_index, float *top_logp, void *workspace,
                                size_t workspace_bytes, void *stream) {
    LogProb l;
    Str z, dz;
    mosa_status st = check_logprob(shape, false, &l, &z, &dz);
    if (st != MOSA_OK) return st;
    if ((st = check_ptrs(shape->dtype, {logits})) != MOSA_OK) return st;
    if (!targets_ok(targets, shape->target64) || !floats_ok({logp, entropy, lse}) ||
        (targets == nullptr && logp != nullptr))
        return MOSA_ERR_INVALID_ARG;
    if (shape->top > 0 && check_ptrs(MOSA_F32, {top_index, top_logp}) != MOSA_OK) return MOSA_ERR_INVALID_ARG;
    if ((st = check_space(workspace, workspace_bytes, logprob_workspace(l))) != MOSA_OK) return st;
    l.z = rows_of(logits, z, shape->dtype);
    l.targets = targets;
    l.logp = logp;
    l.entropy = entropy;
    l.lse = lse;
    l.top_index = top_index;
    l.top_logp = top_logp;
    return of(launch_logprob(l, workspace, (cudaStream_t)stream));
}

mosa_status mosa_token_logprobs_backward(const mosa_logprob_shape *shape, const void *logits,
                                         const void *targets, const float *lse,
                                         const float *entropy, const int32_t *top_index,
                                         const float *dlogp, const float *dentropy,
                                         const float *dlse, const float *dtop_logp, void *dlogits,
                                         void *stream) {
    LogProb l;
    Str z, dz;
    mosa_status st = check_logprob(shape, true, &l, &z, &dz);
    if (st != MOSA_OK) return st;
    if ((st = check_ptrs(shape->dtype, {logits, dlogits})) != MOSA_OK) return st;
    if ((st = check_ptrs(MOSA_F32, {lse})) != MOSA_OK) return st;
    if (!targets_ok(targets, shape->target64) || !floats_ok({entropy, top_index, dlogp, dentropy, dlse, dtop_logp}))
        return MOSA_ERR_INVALID_ARG;
    if ((dlogp != nullptr && targets == nullptr) || (dentropy != nullptr && entropy == nullptr))
        return MOSA_ERR_INVALID_ARG;
    if (shape->top > 0 && (top_index == nullptr || dtop_logp == nullptr)) return MOSA_ERR_INVALID_ARG;
    l.z = rows_of(logits, z, shape->dtype);
    l.dz = rows_of(dlogits, dz, shape->dtype);
    l.targets = targets;
    l.lse = const_cast<float *>(lse);
    l.entropy = const_cast<float *>(entropy);
    l.top_index = const_cast<int32_t *>(top_index);
    l.dlogp = dlogp;
    l.dentropy = dentropy;
    l.dlse = dlse;
    l.dtop = shape->top > 0 ? dtop_logp : nullptr;
    return of(launch_logprob_bwd(l, (cudaStream_t)stream));
}

}  // extern "C"
