// C ABI of the window heads (declared in include/mosa.h): argument checks,
// workspace and dispatch of the norm and rotation of queries and keys, the sliding-window
// attention and the decoding step.
#include <cmath>
#include <cstring>

#include "args.h"
#include "launch.h"
#include "window.h"

namespace mosa {
namespace win {
namespace {

bool hp_ok(int hp) { return hp == 16 || hp == 32 || hp == 64 || hp == 128; }

constexpr int kMaxTokens = 1 << 30;

mosa_status check_heads(int B, int H, int Hkv, int hp, int dtype, bool groups = true) {
    if (B <= 0 || H <= 0 || Hkv <= 0 || hp <= 0) return MOSA_ERR_INVALID_ARG;
    if (groups && H % Hkv != 0) return MOSA_ERR_INVALID_ARG;
    if (dtype != MOSA_F32 && dtype != MOSA_BF16) return MOSA_ERR_INVALID_ARG;
    if (!hp_ok(hp) || B > 65535 || H > 65535) return MOSA_ERR_UNSUPPORTED;
    return MOSA_OK;
}

mosa_status check_rotation(int rotary, int halves, int hp, float theta, float eps) {
    if (rotary < 0 || rotary > hp || rotary % 2 != 0) return MOSA_ERR_INVALID_ARG;
    if (halves != 0 && halves != 1) return MOSA_ERR_INVALID_ARG;
    if (!(theta >= 1.f) || std::isinf(theta) || !(eps >= 0.f) || std::isinf(eps))
        return MOSA_ERR_INVALID_ARG;
    if (halves && rotary % 8 != 0) return MOSA_ERR_UNSUPPORTED;
    return MOSA_OK;
}

mosa_status check_norm(const mosa_qk_shape *s, bool backward, Norm *n) {
    if (s == nullptr) return MOSA_ERR_INVALID_ARG;
    mosa_status st = check_heads(s->B, s->H, s->Hkv, s->hp, s->dtype, /*groups=*/false);
    if (st != MOSA_OK) return st;
    if (s->T <= 0) return MOSA_ERR_INVALID_ARG;
    if (s->T >= kMaxTokens || (long long)s->B * s->T >= (1LL << 31)) return MOSA_ERR_UNSUPPORTED;
    st = check_rotation(s->rotary, s->halves, s->hp, s->theta, s->eps);
    if (st != MOSA_OK) return st;
    *n = Norm{s->B, s->T, s->H, s->Hkv, s->hp, s->dtype == MOSA_BF16, s->rotary, s->halves, s->theta,
              s->eps, {}, {}, {}, {}, {}, {}};
    if (!strides(s->q, s->B, s->T, s->H, &n->q) || !strides(s->k, s->B, s->T, s->Hkv, &n->k) ||
        !strides(s->yq, s->B, s->T, s->H, &n->yq) || !strides(s->yk, s->B, s->T, s->Hkv, &n->yk))
        return MOSA_ERR_INVALID_ARG;
    if (!backward) {
        return output(n->yq, s->B, s->T, s->H, s->hp) && output(n->yk, s->B, s->T, s->Hkv, s->hp)
                   ? MOSA_OK : MOSA_ERR_INVALID_ARG;
    }
    if (!strides(s->dq, s->B, s->T, s->H, &n->dq) || !strides(s->dk, s->B, s->T, s->Hkv, &n->dk))
        return MOSA_ERR_INVALID_ARG;
    return output(n->dq, s->B, s->T, s->H, s->hp) && output(n->dk, s->B, s->T, s->Hkv, s->hp)
               ? MOSA_OK : MOSA_ERR_INVALID_ARG;
}

mosa_status check_window(const mosa_window_shape *s, bool backward, Attn *a) {
    if (s == nullptr) return MOSA_ERR_INVALID_ARG;
    mosa_status st = check_heads(s->B, s->H, s->Hkv, s->hp, s->dtype);
    if (st != MOSA_OK) return st;
    if (s->Tq <= 0 || s->Tq > s->Tk || s->window < 0 || s->sinks < 0) return MOSA_ERR_INVALID_ARG;
    if (!(s->scale >= 0.f) || std::isinf(s->scale)) return MOSA_ERR_INVALID_ARG;
    if (s->Tk >= kMaxTokens || (long long)s->B * s->H * s->Tq >= (1LL << 31)) return MOSA_ERR_UNSUPPORTED;
    *a = Attn{};
    a->B = s->B;
    a->Tq = s->Tq;
    a->Tk = s->Tk;
    a->H = s->H;
    a->Hkv = s->Hkv;
    a->hp = s->hp;
    a->bf16 = s->dtype == MOSA_BF16;
    a->window = s->window == 0 || s->window > s->Tk ? s->Tk : s->window;
    a->sinks = s->sinks < s->Tk ? s->sinks : s->Tk;
    a->scale = s->scale > 0.f ? s->scale : (float)(1.0 / std::sqrt((double)s->hp));
    if (!strides(s->q, s->B, s->Tq, s->H, &a->q) || !strides(s->k, s->B, s->Tk, s->Hkv, &a->k) ||
        !strides(s->v, s->B, s->Tk, s->Hkv, &a->v) || !strides(s->o, s->B, s->Tq, s->H, &a->o))
        return MOSA_ERR_INVALID_ARG;
    if (!backward) return output(a->o, s->B, s->Tq, s->H, s->hp) ? MOSA_OK : MOSA_ERR_INVALID_ARG;
    if (!strides(s->go, s->B, s->Tq, s->H, &a->go) || !strides(s->dq, s->B, s->Tq, s->H, &a->dq) ||
        !strides(s->dk, s->B, s->Tk, s->Hkv, &a->dk) || !strides(s->dv, s->B, s->Tk, s->Hkv, &a->dv))
        return MOSA_ERR_INVALID_ARG;
    return output(a->dq, s->B, s->Tq, s->H, s->hp) && output(a->dk, s->B, s->Tk, s->Hkv, s->hp) &&
                   output(a->dv, s->B, s->Tk, s->Hkv, s->hp)
               ? MOSA_OK : MOSA_ERR_INVALID_ARG;
}

mosa_status check_decode(const mosa_decode_shape *s, Decode *d) {
    if (s == nullptr) return MOSA_ERR_INVALID_ARG;
    mosa_status st = check_heads(s->B, s->H, s->Hkv, s->hp, s->dtype);
    if (st != MOSA_OK) return st;
    if (s->window < 0 || s->sinks < 0 || s->C <= s->sinks) return MOSA_ERR_INVALID_ARG;
    if (s->norm != 0 && s->norm != 1) return MOSA_ERR_INVALID_ARG;
    if (!(s->scale >= 0.f) || std::isinf(s->scale)) return MOSA_ERR_INVALID_ARG;
    if (s->C >= kMaxTokens) return MOSA_ERR_UNSUPPORTED;
    st = check_rotation(s->rotary, s->halves, s->hp, s->theta, s->eps);
    if (st != MOSA_OK) return st;
    const int ring = s->C - s->sinks;
    *d = Decode{s->B, s->C, s->H, s->Hkv, s->hp, s->dtype == MOSA_BF16,
                s->window == 0 || s->window > ring ? ring : s->window, s->sinks, s->norm, s->rotary,
                s->halves, s->scale > 0.f ? s->scale : (float)(1.0 / std::sqrt((double)s->hp)),
                s->theta, s->eps, {}, {}, {}, {}, {}, {}};
    if (!strides(s->q, s->B, 1, s->H, &d->q) || !strides(s->k, s->B, 1, s->Hkv, &d->k) ||
        !strides(s->v, s->B, 1, s->Hkv, &d->v) || !strides(s->o, s->B, 1, s->H, &d->o) ||
        !strides(s->kc, s->B, s->C, s->Hkv, &d->kc) || !strides(s->vc, s->B, s->C, s->Hkv, &d->vc))
        return MOSA_ERR_INVALID_ARG;
    return output(d->o, s->B, 1, s->H, s->hp) && output(d->kc, s->B, s->C, s->Hkv, s->hp) &&
                   output(d->vc, s->B, s->C, s->Hkv, s->hp)
               ? MOSA_OK : MOSA_ERR_INVALID_ARG;
}

mosa_status of(cudaError_t e) { return e == cudaSuccess ? MOSA_OK : MOSA_ERR_CUDA; }

// MOSA_FORCE_SIMT=1 keeps these calls, as the layer's, on the CUDA cores.
bool tensor_cores() { return use_split(); }

// The status word, then the backward's D [B,H,Tq], what the forward's O lost by its rounding
// (bf16 storage) and the backward's partial sums of sink rows.
constexpr size_t kStatusBytes = 256;
size_t rest_at(const Attn &a) {
    return kStatusBytes + ((size_t)a.B * a.H * a.Tq * sizeof(float) + 255) / 256 * 256;
}
size_t partial_at(const Attn &a) {
    return rest_at(a) + (a.bf16 ? ((size_t)a.B * a.H * a.Tq * a.hp * 2 + 255) / 256 * 256 : 0);
}
size_t window_bytes(const Attn &a) {
    return partial_at(a) + window_bwd_bytes(a);
}

}  // namespace
}  // namespace win
}  // namespace mosa

using namespace mosa;
using namespace mosa::win;

extern "C" {

mosa_status mosa_qk_norm_rope(const mosa_qk_shape *shape, const void *q, const void *k,
                              const void *gamma_q, const void *gamma_k,
                              const int32_t *positions, void *yq, void *yk, void *stream) {
    Norm n;
    mosa_status st = check_norm(shape, false, &n);
    if (st != MOSA_OK) return st;
    if ((st = check_ptrs(shape->dtype, {q, k, yq, yk})) != MOSA_OK) return st;
    if (!aligned(gamma_q, shape->dtype) || !aligned(gamma_k, shape->dtype) || !aligned(positions, MOSA_F32))
        return MOSA_ERR_INVALID_ARG;
    return of(launch_norm(n, q, k, gamma_q, gamma_k, positions, yq, yk, (cudaStream_t)stream));
}

size_t mosa_qk_norm_rope_workspace_bytes(const mosa_qk_shape *shape) {
    Norm n;
    return check_norm(shape, true, &n) == MOSA_OK ? norm_workspace(n) : 0;
}

mosa_status mosa_qk_norm_rope_backward(const mosa_qk_shape *shape, const void *q, const void *k,
                                       const void *gamma_q, const void *gamma_k,
                                       const int32_t *positions, const void *dyq,
                                       const void *dyk, void *dq, void *dk, float *dgamma_q,
                                       float *dgamma_k, void *workspace, size_t workspace_bytes,
                                       void *stream) {
    Norm n;
    mosa_status st = check_norm(shape, true, &n);
    if (st != MOSA_OK) return st;
    if ((st = check_ptrs(shape->dtype, {q, k, dyq, dyk, dq, dk})) != MOSA_OK) return st;
    if (!aligned(gamma_q, shape->dtype) || !aligned(gamma_k, shape->dtype) ||
        !aligned(positions, MOSA_F32) || !aligned(dgamma_q, MOSA_F32) || !aligned(dgamma_k, MOSA_F32))
        return MOSA_ERR_INVALID_ARG;
    if ((st = check_space(workspace, workspace_bytes, norm_workspace(n))) != MOSA_OK) return st;
    return of(launch_norm_bwd(n, q, k, gamma_q, gamma_k, positions, dyq, dyk, dq, dk, dgamma_q,
                              dgamma_k, workspace, (cudaStream_t)stream));
}

size_t mosa_window_workspace_bytes(const mosa_window_shape *shape) {
    Attn a;
    return check_window(shape, false, &a) == MOSA_OK ? window_bytes(a) : 0;
}

mosa_status mosa_window_forward(const mosa_window_shape *shape, const void *q, const void *k,
                                const void *v, const int32_t *lens, void *O, float *lse,
                                void *workspace, size_t workspace_bytes, void *stream) {
    Attn a;
    mosa_status st = check_window(shape, false, &a);
    if (st != MOSA_OK) return st;
    if ((st = check_ptrs(shape->dtype, {q, k, v, O})) != MOSA_OK) return st;
    if (!aligned(lens, MOSA_F32) || !aligned(lse, MOSA_F32)) return MOSA_ERR_INVALID_ARG;
    const size_t need = lse != nullptr ? window_bytes(a) : kStatusBytes;
    if ((st = check_space(workspace, workspace_bytes, need)) != MOSA_OK) return st;
    cudaStream_t cs = (cudaStream_t)stream;
    cudaError_t e = cudaSuccess;
    bf16 *rest = lse != nullptr && a.bf16 ? (bf16 *)((char *)workspace + rest_at(a)) : nullptr;
    if (tensor_cores() && tc_window_fwd(a, q, k, v, lens, O, lse, rest, (uint32_t *)workspace, cs, &e))
        return of(e);
    return of(simt_window_fwd(a, q, k, v, lens, O, lse, rest, cs));
}

mosa_status mosa_window_backward(const mosa_window_shape *shape, const void *q, const void *k,
                                 const void *v, const int32_t *lens, const void *O,
                                 const float *lse, const void *dO, void *dq, void *dk, void *dv,
                                 void *workspace, size_t workspace_bytes, void *stream) {
    Attn a;
    mosa_status st = check_window(shape, true, &a);
    if (st != MOSA_OK) return st;
    if ((st = check_ptrs(shape->dtype, {q, k, v, O, dO, dq, dk, dv})) != MOSA_OK) return st;
    if ((st = check_ptrs(MOSA_F32, {lse})) != MOSA_OK) return st;
    if (!aligned(lens, MOSA_F32)) return MOSA_ERR_INVALID_ARG;
    if ((st = check_space(workspace, workspace_bytes, window_bytes(a))) != MOSA_OK) return st;
    float *delta = reinterpret_cast<float *>(static_cast<char *>(workspace) + kStatusBytes);
    cudaStream_t s = (cudaStream_t)stream;
    cudaError_t e = window_delta(a, O, a.bf16 ? (const bf16 *)((const char *)workspace + rest_at(a)) : nullptr, dO,
                                 delta, s);
    if (e != cudaSuccess) return MOSA_ERR_CUDA;
    float *partial = reinterpret_cast<float *>(static_cast<char *>(workspace) + partial_at(a));
    if (tensor_cores() && tc_window_bwd(a, q, k, v, lens, lse, dO, delta, dq, dk, dv, partial,
                                        (uint32_t *)workspace, s, &e))
        return of(e);
    return of(simt_window_bwd(a, q, k, v, lens, lse, dO, delta, dq, dk, dv, partial, s));
}

mosa_status mosa_window_check_status(void *workspace, void *stream) {
    if (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0)
        return MOSA_ERR_WORKSPACE;
    uint32_t v = 0;
    cudaStream_t s = (cudaStream_t)stream;
    if (cudaMemcpyAsync(&v, workspace, sizeof(v), cudaMemcpyDeviceToHost, s) != cudaSuccess ||
        cudaMemsetAsync(workspace, 0, sizeof(v), s) != cudaSuccess ||
        cudaStreamSynchronize(s) != cudaSuccess)
        return MOSA_ERR_CUDA;
    return (v & kStatusTimeout) != 0 ? MOSA_ERR_DEVICE_TIMEOUT : MOSA_OK;
}

size_t mosa_window_decode_workspace_bytes(const mosa_decode_shape *shape) {
    Decode d;
    return check_decode(shape, &d) == MOSA_OK ? decode_workspace(d) : 0;
}

mosa_status mosa_window_decode(const mosa_decode_shape *shape, const void *q, const void *k,
                               const void *v, const void *gamma_q, const void *gamma_k,
                               const int32_t *lens, void *K_cache, void *V_cache, void *O,
                               void *workspace, size_t workspace_bytes, void *stream) {
    Decode d;
    mosa_status st = check_decode(shape, &d);
    if (st != MOSA_OK) return st;
    if ((st = check_ptrs(shape->dtype, {q, k, v, K_cache, V_cache, O})) != MOSA_OK) return st;
    if ((st = check_ptrs(MOSA_F32, {lens})) != MOSA_OK) return st;
    if (!aligned(gamma_q, shape->dtype) || !aligned(gamma_k, shape->dtype)) return MOSA_ERR_INVALID_ARG;
    if ((st = check_space(workspace, workspace_bytes, decode_workspace(d))) != MOSA_OK) return st;
    return of(launch_decode(d, q, k, v, gamma_q, gamma_k, lens, K_cache, V_cache, O, workspace,
                            (cudaStream_t)stream));
}

}  // extern "C"
