// C ABI of the operators around a token mixer: argument validation and dispatch.  All checks run on the
// host before anything is enqueued.
#include "../../include/libloglinear.h"
#include "ll_layer.hpp"

namespace {

constexpr int64_t kMaxTokenStride = int64_t(1) << 24;  // elements; the kernels keep offsets within a tile in 32 bits
constexpr int64_t kMaxChannels = int64_t(1) << 24;
constexpr int64_t kMaxSize = int64_t(1) << 40;         // sequences, tokens of a sequence
constexpr int64_t kMaxElements = int64_t(1) << 44;     // of a tensor: sizes in bytes (up to 2^13 an element) fit 64 bits

bool known_dtype(int32_t d) { return d == LL_F32 || d == LL_BF16; }
bool known_act(int32_t a) { return a == LL_ACT_NONE || a == LL_ACT_SILU; }
bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// B sequences of T tokens of D channels, sizes within what the kernels index.
ll_status check_sizes(int64_t B, int64_t T, int64_t D) {
  if (B < 1 || T < 1 || D < 1) return LL_ERR_BAD_SHAPE;
  if (D >= kMaxChannels || B >= kMaxSize || T >= kMaxSize) return LL_ERR_UNSUPPORTED;
  return T <= kMaxElements / D / B ? LL_OK : LL_ERR_UNSUPPORTED;
}
ll_status check_strides(int64_t batch, int64_t token) {
  if (batch < 0 || token < 0) return LL_ERR_BAD_SHAPE;
  return token < kMaxTokenStride ? LL_OK : LL_ERR_UNSUPPORTED;
}
ll_status check_workspace(const void* ws, size_t bytes, int64_t need) {
  if (need == 0) return LL_OK;
  if (!ws) return LL_ERR_NULL_ARG;
  return bytes >= (size_t)need && aligned(ws, 256) ? LL_OK : LL_ERR_WORKSPACE;
}
ll_status launched(hipError_t e) { return e == hipSuccess ? LL_OK : LL_ERR_HIP; }

#define LL_TRY(expr)                  \
  do {                                \
    const ll_status st_ = (expr);     \
    if (st_ != LL_OK) return st_;     \
  } while (0)

ll_status conv_args(const void* x, int64_t xbs, int64_t xts, const float* weight, int64_t B, int64_t T, int64_t D,
                    int64_t W, int32_t act, int32_t dtype, ll::ConvArgs* a) {
  if (!x || !weight) return LL_ERR_NULL_ARG;
  LL_TRY(check_sizes(B, T, D));
  LL_TRY(check_strides(xbs, xts));
  if (W < 1) return LL_ERR_BAD_SHAPE;
  if (W < 2 || W > 4 || !known_act(act) || !known_dtype(dtype)) return LL_ERR_UNSUPPORTED;
  a->x = {x, xbs, xts};
  a->weight = weight;
  a->B = B, a->T = T, a->D = D, a->W = W, a->act = act, a->dtype = dtype;
  return LL_OK;
}

ll_status scan_args(const ll_scan_inputs* in, ll::ScanArgs* a) {
  if (!in || !in->x || !in->dt || !in->A || !in->B || !in->C) return LL_ERR_NULL_ARG;
  LL_TRY(check_sizes(in->batch, in->T, in->channels));
  if (in->N < 1 || in->groups < 1 || in->channels % in->groups != 0) return LL_ERR_BAD_SHAPE;
  LL_TRY(check_strides(in->x_strides[0], in->x_strides[1]));
  LL_TRY(check_strides(in->dt_strides[0], in->dt_strides[1]));
  LL_TRY(check_strides(in->B_strides[0], in->B_strides[1]));
  LL_TRY(check_strides(in->C_strides[0], in->C_strides[1]));
  if (in->z) LL_TRY(check_strides(in->z_strides[0], in->z_strides[1]));
  if (in->N > ll::kScanMaxN || !known_dtype(in->dtype)) return LL_ERR_UNSUPPORTED;
  a->x = {in->x, in->x_strides[0], in->x_strides[1]};
  a->dt = {in->dt, in->dt_strides[0], in->dt_strides[1]};
  a->Bm = {in->B, in->B_strides[0], in->B_strides[1]};
  a->Cm = {in->C, in->C_strides[0], in->C_strides[1]};
  if (in->z) a->z = {in->z, in->z_strides[0], in->z_strides[1]};
  a->A = in->A, a->skip = in->D, a->dt_bias = in->dt_bias, a->lengths = in->lengths;
  a->B = in->batch, a->T = in->T, a->D = in->channels, a->N = in->N, a->G = in->groups;
  a->softplus = in->delta_softplus != 0, a->dtype = in->dtype;
  return LL_OK;
}

ll_status scan_sizes(int64_t B, int64_t T, int64_t D, int64_t N, int64_t G) {
  LL_TRY(check_sizes(B, T, D));
  if (N < 1 || G < 1 || D % G != 0) return LL_ERR_BAD_SHAPE;
  return N <= ll::kScanMaxN ? LL_OK : LL_ERR_UNSUPPORTED;
}

ll_status norm_args(const void* x, int64_t xbs, int64_t xts, const void* gate, int64_t gbs, int64_t gts, int64_t N,
                    int64_t S, int64_t C, int64_t G, int32_t act, int32_t dtype, ll::NormArgs* a) {
  if (!x) return LL_ERR_NULL_ARG;
  LL_TRY(check_sizes(N, S, C));
  if (G < 1 || C % G != 0) return LL_ERR_BAD_SHAPE;
  LL_TRY(check_strides(xbs, xts));
  if (gate) LL_TRY(check_strides(gbs, gts));
  if (!known_act(act) || !known_dtype(dtype)) return LL_ERR_UNSUPPORTED;
  a->x = {x, xbs, xts};
  if (gate) a->z = {gate, gbs, gts};
  a->N = N, a->S = S, a->C = C, a->G = G, a->act = act, a->dtype = dtype;
  return LL_OK;
}

ll_status decay_sizes(int64_t B, int64_t T, int64_t H, int64_t Hqk, int64_t dk, int64_t dv) {
  if (H < 1 || Hqk < 1 || dk < 1 || dv < 1 || H % Hqk != 0) return LL_ERR_BAD_SHAPE;
  if (H >= kMaxChannels || dk > ll::kDecayMaxWidth || dv > ll::kDecayMaxWidth) return LL_ERR_UNSUPPORTED;
  LL_TRY(check_sizes(B, T, H * (dk > dv ? dk : dv)));
  return B <= kMaxElements / (H * dk * dv) ? LL_OK : LL_ERR_UNSUPPORTED;
}

ll_status decay_args(const ll_decay_inputs* in, ll::DecayArgs* a) {
  if (!in || !in->q || !in->k || !in->v || !in->log_decay) return LL_ERR_NULL_ARG;
  LL_TRY(decay_sizes(in->batch, in->T, in->heads, in->qk_heads, in->d_k, in->d_v));
  LL_TRY(check_strides(in->q_strides[0], in->q_strides[1]));
  LL_TRY(check_strides(in->k_strides[0], in->k_strides[1]));
  LL_TRY(check_strides(in->v_strides[0], in->v_strides[1]));
  if (!known_dtype(in->dtype)) return LL_ERR_UNSUPPORTED;
  a->q = {in->q, in->q_strides[0], in->q_strides[1]};
  a->k = {in->k, in->k_strides[0], in->k_strides[1]};
  a->v = {in->v, in->v_strides[0], in->v_strides[1]};
  a->log_decay = in->log_decay, a->lengths = in->lengths;
  a->B = in->batch, a->T = in->T, a->H = in->heads, a->Hqk = in->qk_heads, a->dk = in->d_k, a->dv = in->d_v;
  a->scale = in->scale, a->dtype = in->dtype;
  return LL_OK;
}

// x [M, K] and W [N, K] to [M, N].
ll_status projection_sizes(int64_t M, int64_t K, int64_t N, int32_t act, int32_t dtype) {
  LL_TRY(check_sizes(M, 1, K));
  LL_TRY(check_sizes(M, 1, N));
  LL_TRY(check_sizes(N, 1, K));
  return known_act(act) && known_dtype(dtype) ? LL_OK : LL_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" {

ll_status ll_causal_conv_fwd(const void* x, int64_t x_batch_stride, int64_t x_token_stride, const float* weight,
                             const float* bias, const void* initial_state, void* final_state, const int32_t* lengths,
                             void* y, int64_t B, int64_t T, int64_t D, int64_t W, int32_t act, int32_t dtype,
                             void* stream) {
  ll::ConvArgs a = {};
  LL_TRY(conv_args(x, x_batch_stride, x_token_stride, weight, B, T, D, W, act, dtype, &a));
  if (!y) return LL_ERR_NULL_ARG;
  if (!ll::conv_launchable(a, false)) return LL_ERR_UNSUPPORTED;
  a.bias = bias, a.state = initial_state, a.new_state = final_state, a.lengths = lengths, a.y = y;
  return launched(ll::launch_conv_fwd(a, static_cast<hipStream_t>(stream)));
}

ll_status ll_causal_conv_step(const void* x, int64_t x_batch_stride, const float* weight, const float* bias,
                              const void* state, void* new_state, void* y, int64_t B, int64_t D, int64_t W,
                              int32_t act, int32_t dtype, void* stream) {
  ll::ConvArgs a = {};
  LL_TRY(conv_args(x, x_batch_stride, 0, weight, B, 1, D, W, act, dtype, &a));
  if (!state || !new_state || !y) return LL_ERR_NULL_ARG;
  if (!ll::conv_launchable(a, false)) return LL_ERR_UNSUPPORTED;
  a.bias = bias, a.state = state, a.new_state = new_state, a.y = y;
  return launched(ll::launch_conv_step(a, static_cast<hipStream_t>(stream)));
}

size_t ll_causal_conv_bwd_workspace_size(int32_t dtype, int64_t B, int64_t T, int64_t D, int64_t W) {
  if (check_sizes(B, T, D) != LL_OK || W < 2 || W > 4 || !known_dtype(dtype)) return 0;
  return (size_t)ll::conv_bwd_workspace(B, T, D, W, dtype);
}

ll_status ll_causal_conv_bwd(const void* x, int64_t x_batch_stride, int64_t x_token_stride, const float* weight,
                             const float* bias, const void* initial_state, const int32_t* lengths, const void* d_y,
                             const void* d_final_state, void* dx, float* dweight, float* dbias,
                             void* d_initial_state, int64_t B, int64_t T, int64_t D, int64_t W, int32_t act,
                             int32_t dtype, void* workspace, size_t workspace_bytes, void* stream) {
  ll::ConvArgs a = {};
  LL_TRY(conv_args(x, x_batch_stride, x_token_stride, weight, B, T, D, W, act, dtype, &a));
  if (!d_y || !dx || !dweight) return LL_ERR_NULL_ARG;
  if (!ll::conv_launchable(a, true)) return LL_ERR_UNSUPPORTED;
  LL_TRY(check_workspace(workspace, workspace_bytes, ll::conv_bwd_workspace(B, T, D, W, dtype)));
  a.bias = bias, a.state = initial_state, a.lengths = lengths;
  const ll::ConvGrads g = {d_y, d_final_state, dx, dweight, dbias, d_initial_state, workspace};
  return launched(ll::launch_conv_bwd(a, g, static_cast<hipStream_t>(stream)));
}

size_t ll_selective_scan_states_bytes(int64_t B, int64_t T, int64_t D, int64_t N) {
  return scan_sizes(B, T, D, N, 1) == LL_OK ? (size_t)ll::scan_states_bytes(B, T, D, N) : 0;
}

size_t ll_selective_scan_workspace_size(int64_t B, int64_t T, int64_t D, int64_t N, int64_t groups,
                                        int32_t backward) {
  if (scan_sizes(B, T, D, N, groups) != LL_OK) return 0;
  return (size_t)(backward ? ll::scan_bwd_workspace(B, T, D, N, groups) : ll::scan_fwd_workspace(B, T, D, N, groups));
}

ll_status ll_selective_scan_fwd(const ll_scan_inputs* in, const float* initial_state, void* y, float* final_state,
                                float* states, void* workspace, size_t workspace_bytes, void* stream) {
  ll::ScanArgs a = {};
  LL_TRY(scan_args(in, &a));
  if (!y) return LL_ERR_NULL_ARG;
  if (!ll::scan_fwd_launchable(a)) return LL_ERR_UNSUPPORTED;
  LL_TRY(check_workspace(workspace, workspace_bytes, ll::scan_fwd_workspace(a.B, a.T, a.D, a.N, a.G)));
  if (!aligned(states, 16)) return LL_ERR_WORKSPACE;
  a.h0 = initial_state, a.h_final = final_state, a.states = states, a.y = y, a.workspace = workspace;
  return launched(ll::launch_scan_fwd(a, static_cast<hipStream_t>(stream)));
}

ll_status ll_selective_scan_step(const ll_scan_inputs* in, const float* state, float* new_state, void* y,
                                 void* stream) {
  ll::ScanArgs a = {};
  LL_TRY(scan_args(in, &a));
  if (!state || !new_state || !y) return LL_ERR_NULL_ARG;
  if (a.T != 1 || a.lengths) return LL_ERR_BAD_SHAPE;
  if (!ll::scan_step_launchable(a)) return LL_ERR_UNSUPPORTED;
  a.h0 = state, a.h_final = new_state, a.y = y;
  return launched(ll::launch_scan_step(a, static_cast<hipStream_t>(stream)));
}

ll_status ll_selective_scan_bwd(const ll_scan_inputs* in, const float* states, const void* d_y,
                                const float* d_final_state, void* dx, void* ddt, void* dz, float* dA, void* dB,
                                void* dC, float* dD, float* ddt_bias, float* d_initial_state, void* workspace,
                                size_t workspace_bytes, void* stream) {
  ll::ScanArgs a = {};
  LL_TRY(scan_args(in, &a));
  if (!states || !d_y || !dx || !ddt || !dA || !dB || !dC || (a.z.p && !dz)) return LL_ERR_NULL_ARG;
  if (!ll::scan_bwd_launchable(a)) return LL_ERR_UNSUPPORTED;
  LL_TRY(check_workspace(workspace, workspace_bytes, ll::scan_bwd_workspace(a.B, a.T, a.D, a.N, a.G)));
  if (!aligned(states, 16)) return LL_ERR_WORKSPACE;
  a.states = const_cast<float*>(states), a.workspace = workspace;
  const ll::ScanGrads g = {d_y, d_final_state, dx, ddt, a.z.p ? dz : nullptr, dA, dB, dC, dD, ddt_bias, d_initial_state};
  return launched(ll::launch_scan_bwd(a, g, static_cast<hipStream_t>(stream)));
}

size_t ll_group_norm_workspace_size(int32_t dtype, int64_t N, int64_t S, int64_t C, int64_t groups,
                                    int32_t backward) {
  if (check_sizes(N, S, C) != LL_OK || groups < 1 || C % groups != 0 || !known_dtype(dtype)) return 0;
  return (size_t)ll::norm_workspace(N, S, C, groups, dtype, backward != 0);
}

ll_status ll_group_norm_fwd(const void* x, int64_t x_batch_stride, int64_t x_token_stride, const void* gate,
                            int64_t gate_batch_stride, int64_t gate_token_stride, const float* weight,
                            const float* bias, void* y, float* stats, int64_t N, int64_t S, int64_t C,
                            int64_t groups, float eps, int32_t act, int32_t dtype, void* workspace,
                            size_t workspace_bytes, void* stream) {
  ll::NormArgs a = {};
  LL_TRY(norm_args(x, x_batch_stride, x_token_stride, gate, gate_batch_stride, gate_token_stride, N, S, C, groups, act,
                   dtype, &a));
  if (!y) return LL_ERR_NULL_ARG;
  if (!ll::norm_launchable(a, false)) return LL_ERR_UNSUPPORTED;
  LL_TRY(check_workspace(workspace, workspace_bytes, ll::norm_workspace(N, S, C, groups, dtype, false)));
  if (!aligned(stats, 8)) return LL_ERR_WORKSPACE;
  a.weight = weight, a.bias = bias, a.y = y, a.stats = stats, a.eps = eps, a.workspace = workspace;
  return launched(ll::launch_norm_fwd(a, static_cast<hipStream_t>(stream)));
}

ll_status ll_group_norm_bwd(const void* x, int64_t x_batch_stride, int64_t x_token_stride, const void* gate,
                            int64_t gate_batch_stride, int64_t gate_token_stride, const float* weight,
                            const float* bias, const float* stats, const void* d_y, void* dx, void* dgate,
                            float* dweight, float* dbias, int64_t N, int64_t S, int64_t C, int64_t groups,
                            int32_t act, int32_t dtype, void* workspace, size_t workspace_bytes, void* stream) {
  ll::NormArgs a = {};
  LL_TRY(norm_args(x, x_batch_stride, x_token_stride, gate, gate_batch_stride, gate_token_stride, N, S, C, groups, act,
                   dtype, &a));
  if (!stats || !d_y || !dx || (gate && !dgate)) return LL_ERR_NULL_ARG;
  if (!ll::norm_launchable(a, true)) return LL_ERR_UNSUPPORTED;
  LL_TRY(check_workspace(workspace, workspace_bytes, ll::norm_workspace(N, S, C, groups, dtype, true)));
  if (!aligned(stats, 8)) return LL_ERR_WORKSPACE;
  a.weight = weight, a.bias = bias, a.stats = const_cast<float*>(stats), a.workspace = workspace;
  const ll::NormGrads g = {d_y, dx, gate ? dgate : nullptr, dweight, dbias};
  return launched(ll::launch_norm_bwd(a, g, static_cast<hipStream_t>(stream)));
}

size_t ll_decay_attention_workspace_size(int64_t B, int64_t T, int64_t H, int64_t H_qk, int64_t d_k, int64_t d_v,
                                         int32_t backward) {
  if (decay_sizes(B, T, H, H_qk, d_k, d_v) != LL_OK) return 0;
  return (size_t)ll::decay_workspace(B, T, H, H_qk, d_k, d_v, backward != 0);
}

size_t ll_decay_attention_states_bytes(int64_t B, int64_t T, int64_t H, int64_t d_k, int64_t d_v) {
  return decay_sizes(B, T, H, H, d_k, d_v) == LL_OK ? (size_t)ll::decay_states_bytes(B, T, H, d_k, d_v) : 0;
}

ll_status ll_decay_attention_fwd(const ll_decay_inputs* in, const float* initial_state, void* o, float* final_state,
                                 float* states, void* workspace, size_t workspace_bytes, void* stream) {
  ll::DecayArgs a = {};
  LL_TRY(decay_args(in, &a));
  if (!o) return LL_ERR_NULL_ARG;
  if (!ll::decay_launchable(a, false)) return LL_ERR_UNSUPPORTED;
  // states of the caller's serve as workspace
  if (!states) LL_TRY(check_workspace(workspace, workspace_bytes, ll::decay_workspace(a.B, a.T, a.H, a.Hqk, a.dk, a.dv, false)));
  if (!aligned(states, 16)) return LL_ERR_WORKSPACE;
  a.initial = initial_state, a.final_state = final_state, a.states = states, a.o = o, a.workspace = workspace;
  return launched(ll::launch_decay_fwd(a, static_cast<hipStream_t>(stream)));
}

ll_status ll_decay_attention_step(const ll_decay_inputs* in, const float* state, float* new_state, void* o,
                                  void* stream) {
  ll::DecayArgs a = {};
  LL_TRY(decay_args(in, &a));
  if (!state || !new_state || !o) return LL_ERR_NULL_ARG;
  if (a.T != 1 || a.lengths) return LL_ERR_BAD_SHAPE;
  if (!ll::decay_step_launchable(a)) return LL_ERR_UNSUPPORTED;
  a.initial = state, a.final_state = new_state, a.o = o;
  return launched(ll::launch_decay_step(a, static_cast<hipStream_t>(stream)));
}

ll_status ll_decay_attention_bwd(const ll_decay_inputs* in, const float* states, const void* d_o,
                                 const float* d_final_state, void* dq, void* dk, void* dv, float* d_initial_state,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  ll::DecayArgs a = {};
  LL_TRY(decay_args(in, &a));
  if (!states || !d_o || !dq || !dk || !dv) return LL_ERR_NULL_ARG;
  if (!ll::decay_launchable(a, true)) return LL_ERR_UNSUPPORTED;
  LL_TRY(check_workspace(workspace, workspace_bytes, ll::decay_workspace(a.B, a.T, a.H, a.Hqk, a.dk, a.dv, true)));
  if (!aligned(states, 16)) return LL_ERR_WORKSPACE;
  a.states = const_cast<float*>(states), a.workspace = workspace;
  const ll::DecayGrads g = {d_o, d_final_state, dq, dk, dv, d_initial_state};
  return launched(ll::launch_decay_bwd(a, g, static_cast<hipStream_t>(stream)));
}

size_t ll_projection_workspace_size(int32_t dtype, int64_t M, int64_t K, int64_t N, int32_t act, int32_t backward) {
  if (projection_sizes(M, K, N, act, dtype) != LL_OK) return 0;
  return (size_t)ll::projection_workspace(M, K, N, act, dtype, backward != 0);
}

ll_status ll_projection_fwd(const void* x, int64_t x_stride, const void* weight, const float* bias,
                            const void* residual, int64_t residual_stride, void* y, float* pre, int64_t M, int64_t K,
                            int64_t N, int32_t act, int32_t dtype, void* workspace, size_t workspace_bytes,
                            void* stream) {
  if (!x || !weight || !y) return LL_ERR_NULL_ARG;
  LL_TRY(projection_sizes(M, K, N, act, dtype));
  LL_TRY(check_strides(0, x_stride));
  if (residual) LL_TRY(check_strides(0, residual_stride));
  if (!ll::projection_launchable(M, K, N, act, dtype, false)) return LL_ERR_UNSUPPORTED;
  LL_TRY(check_workspace(workspace, workspace_bytes, ll::projection_workspace(M, K, N, act, dtype, false)));
  const ll::ProjArgs a = {x, x_stride, weight, bias, residual, residual_stride, y, pre, M, K, N, act, dtype, workspace};
  return launched(ll::launch_projection_fwd(a, static_cast<hipStream_t>(stream)));
}

ll_status ll_projection_bwd(const void* x, int64_t x_stride, const void* weight, const float* pre, const void* d_y,
                            void* dx, void* dweight, float* dbias, int64_t M, int64_t K, int64_t N, int32_t act,
                            int32_t dtype, void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !weight || !d_y) return LL_ERR_NULL_ARG;
  LL_TRY(projection_sizes(M, K, N, act, dtype));
  LL_TRY(check_strides(0, x_stride));
  if (act != LL_ACT_NONE && !pre) return LL_ERR_NULL_ARG;
  if (!ll::projection_launchable(M, K, N, act, dtype, true)) return LL_ERR_UNSUPPORTED;
  LL_TRY(check_workspace(workspace, workspace_bytes, ll::projection_workspace(M, K, N, act, dtype, true)));
  ll::ProjArgs a = {};
  a.x = x, a.x_stride = x_stride, a.weight = weight, a.pre = const_cast<float*>(pre), a.M = M, a.K = K, a.N = N;
  a.act = act, a.dtype = dtype, a.workspace = workspace;
  const ll::ProjGrads g = {d_y, dx, dweight, dbias};
  return launched(ll::launch_projection_bwd(a, g, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
