// C ABI of the operators on either side of the norms and sums: LayerNorm, the
// head's losses, orthogonalised updates (part of api.cpp, whose helpers it uses).
#pragma once

namespace {

constexpr int64_t MAX_ROWS = ((int64_t)1 << 31) - (1 << 16);  // rows are counted in 32 bits

// Rows of w elements, ld apart, of a matrix of B*T rows.
dp_status_t check_rows(int B, int T, int w, dp_dtype_t dt, const char* width) {
  if (B <= 0 || T <= 0 || w <= 0) return fail(DP_EINVAL, "B, T and %s must be positive", width);
  if (!dtype_ok(dt)) return fail(DP_EINVAL, "unknown dtype %d", (int)dt);
  if ((int64_t)B * T > MAX_ROWS)
    return fail(DP_EUNSUPPORTED, "B*T = %lld exceeds 2^31 - 2^16", (long long)((int64_t)B * T));
  return DP_OK;
}

struct LnWorkspace {
  dpg::LnPlan plan;
  size_t sq, total;  // offset of the partial squares; bytes in all
};
LnWorkspace ln_workspace(int B, int T, int d) {
  LnWorkspace w;
  w.plan = dpg::ln_plan(B, T, d, true);
  w.sq = w.total = 0;
  if (w.plan.ranges > 1) {
    w.sq = align_up((size_t)B * w.plan.ranges * 2 * (size_t)d * 4);
    w.total = w.sq + align_up((size_t)B * w.plan.chunks * 4);
  }
  return w;
}

// Preference loss scratch: log p (double), statistics and slopes of the rows.
struct PrefLayout {
  size_t stat, slope, total;
};
PrefLayout pref_layout(int B, int T) {
  const size_t rows = (size_t)B * T;
  PrefLayout l;
  l.stat = align_up(rows * 8);
  l.slope = l.stat + align_up(rows * sizeof(dpg::RowStat));
  l.total = l.slope + align_up((size_t)B * 4);
  return l;
}

constexpr int MAX_LOGITS = 1 << 30;  // columns are counted in 32 bits

dp_status_t check_logits(const void* Z, int64_t ldz, const int32_t* targets, int B, int T, int V,
                         dp_dtype_t dt) {
  if (!Z || !targets) return fail(DP_EINVAL, "Z or targets is NULL");
  dp_status_t st = check_rows(B, T, V, dt, "V");
  if (st != DP_OK) return st;
  if (V > MAX_LOGITS) return fail(DP_EUNSUPPORTED, "V = %d exceeds 2^30", V);
  if (ldz < V) return fail(DP_EINVAL, "ldz < V");
  return DP_OK;
}

// The gradient may replace the logits, but not overlap them in another layout.
dp_status_t check_in_place(const void* Z, int64_t ldz, const void* Gz, int64_t ldg) {
  if (Gz == Z && ldg != ldz) return fail(DP_EINVAL, "in place, ldg must equal ldz");
  return DP_OK;
}

inline int ns_padded(int x) { return (int)ceil_div(x, dpg::NS_TILE) * dpg::NS_TILE; }
// Planes of a matrix's operands. Few rows average few roundings: of 16 x 16 a bf16 result's
// products alone are 2.0e-3 off with one plane, of 64 x 64 1.5e-3, of 200 x 200 1.1e-3, of 512 x 1024 0.9e-3.
inline int ns_planes(const dp_matrix_t& m, dp_dtype_t out_dt) {
  return out_dt == DP_BF16 && std::min(m.rows, m.cols) > 64 ? 1 : 2;
}

// The launches of a group: up to NS_MAX_MATS matrices each, from *next on; those of one and of
// two planes, and the small ones (dpg::ns_small), apart.
dpg::NsArgs ns_batch(const dp_matrix_t* m, int n, dp_dtype_t out_dt, int pl, bool small, int* next) {
  dpg::NsArgs a{};
  for (; *next < n && a.n < dpg::NS_MAX_MATS; ++*next) {
    const dp_matrix_t& x = m[*next];
    if (ns_planes(x, out_dt) != pl || dpg::ns_small(x.rows, x.cols, pl) != small) continue;
    dpg::NsMat& M = a.M[a.n++];
    M.G = x.G; M.out = x.out; M.ldg = x.ldg; M.ldo = x.ldo;
    M.rows = x.rows; M.cols = x.cols; M.scale = x.scale;
    const int s = std::min(x.rows, x.cols), l = std::max(x.rows, x.cols);
    M.mp = small ? (int)ceil_div(s, 32) * 32 : ns_padded(s);
    M.np = small ? (int)ceil_div(l, 32) * 32 : ns_padded(l);
  }
  return a;
}

// Bytes of a launch's matrices, and of the parts of split sums behind them.
size_t ns_batch_bytes(const dpg::NsArgs& a, int pl) {
  size_t bytes = align_up(dpg::ns_part_bytes(a, pl));
  for (int l = 0; l < a.n; ++l) bytes += align_up(dpg::ns_bytes(a.M[l].mp, a.M[l].np, pl));
  return bytes;
}

// Checks the sizes and strides; *bytes gets the workspace the group needs (its
// launches follow one another, so they share it).
dp_status_t check_matrices(const dp_matrix_t* m, int n, dp_dtype_t in_dt, dp_dtype_t out_dt,
                           size_t* bytes) {
  if (!m || n <= 0) return fail(DP_EINVAL, "no matrices");
  if (!dtype_ok(in_dt)) return fail(DP_EINVAL, "unknown dtype %d", (int)in_dt);
  if (!dtype_ok(out_dt)) return fail(DP_EINVAL, "unknown dtype %d", (int)out_dt);
  for (int l = 0; l < n; ++l) {
    const dp_matrix_t& x = m[l];
    if (x.rows <= 0 || x.cols <= 0) return fail(DP_EINVAL, "matrix %d: empty", l);
    if (x.rows > dpg::NS_MAX_SIDE || x.cols > dpg::NS_MAX_SIDE)
      return fail(DP_EUNSUPPORTED, "matrix %d: a side exceeds %d", l, dpg::NS_MAX_SIDE);
    if (x.ldg < x.cols || x.ldo < x.cols)
      return fail(DP_EINVAL, "matrix %d: row stride smaller than its columns", l);
    if ((int64_t)ns_padded(x.rows) * ns_padded(x.cols) >= dpg::NS_MAX_SIZE)
      return fail(DP_EUNSUPPORTED, "matrix %d: 2^30 elements or more", l);
  }
  *bytes = 0;
  for (int pl = 1; pl <= 2; ++pl)
    for (int next = 0; next < n;) {
      const dpg::NsArgs a = ns_batch(m, n, out_dt, pl, false, &next);
      if (a.n) *bytes = std::max(*bytes, ns_batch_bytes(a, pl));
    }
  return DP_OK;
}

}  // namespace

extern "C" {

dp_status_t dp_layernorm_forward(const void* x, int64_t ldx, const void* gain, const void* bias,
                                 dp_dtype_t param_dt, int B, int T, int d, dp_dtype_t dt,
                                 float eps, void* y, int64_t ldy, float* mean, float* rstd,
                                 void* stream) {
  if (!x || !y) return fail(DP_EINVAL, "x or y is NULL");
  dp_status_t st = check_rows(B, T, d, dt, "d");
  if (st != DP_OK) return st;
  if (!dtype_ok(param_dt)) return fail(DP_EINVAL, "unknown dtype %d", (int)param_dt);
  if (d > dpg::LN_MAX_D) return fail(DP_EUNSUPPORTED, "d = %d exceeds %d", d, dpg::LN_MAX_D);
  if (ldx < d || ldy < d) return fail(DP_EINVAL, "row stride smaller than d");
  if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(DP_EINVAL, "eps must be >= 0");
  if (y == x && ldy != ldx) return fail(DP_EINVAL, "in place, ldy must equal ldx");
  dpg::LnForwardArgs a{};
  a.x = x; a.gain = gain; a.bias = bias; a.y = y; a.mean = mean; a.rstd = rstd;
  a.ldx = ldx; a.ldy = ldy; a.rows = (int64_t)B * T;
  a.d = d; a.param_dt = kdt(param_dt); a.eps = eps;
  return hip_status(dpg::launch_ln_forward(a, kdt(dt), as_stream(stream)), "layernorm launch");
}

size_t dp_layernorm_backward_workspace(int B, int T, int d) {
  if (B <= 0 || T <= 0 || d <= 0 || d > dpg::LN_MAX_D || (int64_t)B * T > MAX_ROWS) return 0;
  return ln_workspace(B, T, d).total;
}

dp_status_t dp_layernorm_backward(const void* gy, int64_t ldgy, const void* x, int64_t ldx,
                                  const void* gain, dp_dtype_t param_dt, const float* mean,
                                  const float* rstd, int B, int T, int d, dp_dtype_t dt, void* dx,
                                  int64_t lddx, int accumulate_dx, float* dgain, float* dbias,
                                  float* norm2, int accumulate, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  if (!gy || !x || !mean || !rstd) return fail(DP_EINVAL, "gy, x, mean or rstd is NULL");
  if (!dx && !dgain && !dbias) return fail(DP_EINVAL, "dx, dgain and dbias are all NULL");
  if (norm2 && !dgain && !dbias)
    return fail(DP_EINVAL, "norm2 is the squared norm of dgain and dbias: both are NULL");
  dp_status_t st = check_rows(B, T, d, dt, "d");
  if (st != DP_OK) return st;
  if (!dtype_ok(param_dt)) return fail(DP_EINVAL, "unknown dtype %d", (int)param_dt);
  if (d > dpg::LN_MAX_D) return fail(DP_EUNSUPPORTED, "d = %d exceeds %d", d, dpg::LN_MAX_D);
  if (ldgy < d || ldx < d || (dx && lddx < d)) return fail(DP_EINVAL, "row stride smaller than d");
  if (dx && ((dx == gy && lddx != ldgy) || (dx == x && lddx != ldx)))
    return fail(DP_EINVAL, "in place, lddx must equal the operand's row stride");
  const bool grads = dgain || dbias;
  dpg::LnBackwardArgs a{};
  LnWorkspace w{dpg::ln_plan(B, T, d, false), 0, 0};
  if (grads) w = ln_workspace(B, T, d);
  if (w.total) {
    if (!workspace || workspace_bytes < w.total)
      return fail(DP_EINVAL, "workspace of %zu bytes needed", w.total);
    if (!aligned16(workspace)) return fail(DP_EINVAL, "workspace must be 16-byte aligned");
    a.ws = static_cast<float*>(workspace);
    a.sq = reinterpret_cast<float*>(static_cast<char*>(workspace) + w.sq);
  }
  a.gy = gy; a.x = x; a.gain = gain; a.mean = mean; a.rstd = rstd;
  a.dx = dx; a.dgain = dgain; a.dbias = dbias; a.norm2 = norm2;
  a.ldgy = ldgy; a.ldx = ldx; a.lddx = lddx;
  a.B = B; a.T = T; a.d = d; a.param_dt = kdt(param_dt);
  a.ranges = w.plan.ranges; a.span = w.plan.span; a.chunks = w.plan.chunks;
  a.accumulate_dx = accumulate_dx ? 1 : 0; a.accumulate = accumulate ? 1 : 0;
  return hip_status(dpg::launch_ln_backward(a, kdt(dt), as_stream(stream)),
                    "layernorm backward launch");
}

dp_status_t dp_token_logprobs(const void* Z, int64_t ldz, const int32_t* targets, int B, int T,
                              int V, dp_dtype_t dt, float* logp, float* lse, void* stream) {
  dp_status_t st = check_logits(Z, ldz, targets, B, T, V, dt);
  if (st != DP_OK) return st;
  if (!logp) return fail(DP_EINVAL, "logp is NULL");
  dpg::LossArgs a{};
  a.Z = Z; a.ldz = ldz; a.targets = targets; a.logp = logp; a.lse = lse;
  a.rows = (int64_t)B * T; a.V = V; a.T = T;
  return hip_status(dpg::launch_token_logprobs(a, kdt(dt), as_stream(stream)),
                    "token_logprobs launch");
}

dp_status_t dp_cross_entropy(const void* Z, int64_t ldz, const int32_t* targets, const float* w,
                             int B, int T, int V, dp_dtype_t dt, float* logp, void* Gz,
                             int64_t ldg, void* stream) {
  dp_status_t st = check_logits(Z, ldz, targets, B, T, V, dt);
  if (st != DP_OK) return st;
  if (!w || !Gz) return fail(DP_EINVAL, "w or Gz is NULL");
  if (ldg < V) return fail(DP_EINVAL, "ldg < V");
  st = check_in_place(Z, ldz, Gz, ldg);
  if (st != DP_OK) return st;
  dpg::LossArgs a{};
  a.Z = Z; a.ldz = ldz; a.targets = targets; a.w = w; a.logp = logp; a.Gz = Gz; a.ldg = ldg;
  a.rows = (int64_t)B * T; a.V = V; a.T = T;
  return hip_status(dpg::launch_cross_entropy(a, kdt(dt), as_stream(stream)),
                    "cross_entropy launch");
}

size_t dp_preference_loss_workspace(int B, int T) {
  if (B <= 0 || T <= 0 || (int64_t)B * T > MAX_ROWS) return 0;
  return pref_layout(B, T).total;
}

dp_status_t dp_preference_loss(const void* Z, int64_t ldz, const int32_t* targets, int split,
                               const float* ref_logp, float beta, float label_smoothing, int B,
                               int T, int V, dp_dtype_t dt, float* loss, float* rewards,
                               float* logp, void* Gz, int64_t ldg, void* workspace,
                               size_t workspace_bytes, void* stream) {
  dp_status_t st = check_logits(Z, ldz, targets, B, T, V, dt);
  if (st != DP_OK) return st;
  if (!loss) return fail(DP_EINVAL, "loss is NULL");
  if (split < 0 || split > T) return fail(DP_EINVAL, "split = %d is not in [0, T]", split);
  if (!(beta > 0.f) || !std::isfinite(beta)) return fail(DP_EINVAL, "beta must be positive");
  if (!(label_smoothing >= 0.f) || !(label_smoothing < 0.5f))
    return fail(DP_EINVAL, "label_smoothing must be in [0, 0.5)");
  if (Gz) {
    if (ldg < V) return fail(DP_EINVAL, "ldg < V");
    st = check_in_place(Z, ldz, Gz, ldg);
    if (st != DP_OK) return st;
  }
  const PrefLayout l = pref_layout(B, T);
  if (!workspace || workspace_bytes < l.total)
    return fail(DP_EINVAL, "workspace of %zu bytes needed", l.total);
  if (!aligned16(workspace)) return fail(DP_EINVAL, "workspace must be 16-byte aligned");
  char* ws = static_cast<char*>(workspace);
  hipStream_t s = as_stream(stream);
  dpg::LossArgs a{};
  a.Z = Z; a.ldz = ldz; a.targets = targets; a.logp = logp; a.Gz = Gz; a.ldg = ldg;
  a.logp64 = reinterpret_cast<double*>(ws);
  a.stat = reinterpret_cast<dpg::RowStat*>(ws + l.stat);
  a.w = reinterpret_cast<float*>(ws + l.slope);
  a.V = V; a.T = T; a.split = split;
  a.rows = (int64_t)B * T;
  st = hip_status(dpg::launch_token_logprobs(a, kdt(dt), s), "token_logprobs launch");
  if (st != DP_OK) return st;
  dpg::PreferenceArgs p{};
  p.targets = targets; p.logp = a.logp64; p.ref = ref_logp; p.loss = loss; p.rewards = rewards;
  p.slope = reinterpret_cast<float*>(ws + l.slope);
  p.T = T; p.V = V; p.split = split; p.beta = beta; p.smoothing = label_smoothing;
  st = hip_status(dpg::launch_preference(p, B, s), "preference launch");
  if (st != DP_OK || !Gz) return st;
  return hip_status(dpg::launch_logit_grads(a, kdt(dt), s), "logit_grads launch");
}

size_t dp_orthogonalize_workspace(const dp_matrix_t* matrices, int n, dp_dtype_t out_dt) {
  size_t bytes = 0;
  return check_matrices(matrices, n, DP_F32, out_dt, &bytes) == DP_OK ? bytes : 0;
}

dp_status_t dp_orthogonalize_grouped(const dp_matrix_t* matrices, int n, dp_dtype_t in_dt,
                                     dp_dtype_t out_dt, const float* coef, int steps, float eps,
                                     int accumulate, void* workspace, size_t workspace_bytes,
                                     void* stream) {
  size_t need = 0;
  dp_status_t st = check_matrices(matrices, n, in_dt, out_dt, &need);
  if (st != DP_OK) return st;
  if (!coef) return fail(DP_EINVAL, "coef is NULL");
  if (steps < 1 || steps > dpg::NS_MAX_STEPS)
    return fail(DP_EINVAL, "steps = %d is not in [1, %d]", steps, dpg::NS_MAX_STEPS);
  for (int k = 0; k < 3 * steps; ++k)
    if (!std::isfinite(coef[k])) return fail(DP_EINVAL, "coef[%d] is not finite", k);
  if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(DP_EINVAL, "eps must be >= 0");
  for (int l = 0; l < n; ++l) {
    if (!matrices[l].G || !matrices[l].out) return fail(DP_EINVAL, "matrix %d: G or out is NULL", l);
    if (!std::isfinite(matrices[l].scale)) return fail(DP_EINVAL, "matrix %d: scale is not finite", l);
  }
  if (need && (!workspace || workspace_bytes < need))
    return fail(DP_EINVAL, "workspace of %zu bytes needed", need);
  if (need && !aligned16(workspace)) return fail(DP_EINVAL, "workspace must be 16-byte aligned");
  for (int pl = 1; pl <= 2; ++pl)
    for (int big = 0; big <= 1; ++big)
      for (int next = 0; next < n;) {
        dpg::NsArgs a = ns_batch(matrices, n, out_dt, pl, !big, &next);
        if (a.n == 0) break;
        a.out_dt = kdt(out_dt); a.accumulate = accumulate ? 1 : 0; a.eps = eps;
        hipError_t e;
        if (big) {
          char* ws = static_cast<char*>(workspace);
          for (int l = 0; l < a.n; ++l) {
            a.M[l].ws = ws;
            ws += align_up(dpg::ns_bytes(a.M[l].mp, a.M[l].np, pl));
          }
          a.part = reinterpret_cast<float*>(ws);
          e = dpg::launch_orthogonalize(a, kdt(in_dt), pl, coef, steps, as_stream(stream));
        } else {
          e = dpg::launch_orthogonalize_small(a, kdt(in_dt), pl, coef, steps, as_stream(stream));
        }
        st = hip_status(e, "orthogonalize launch");
        if (st != DP_OK) return st;
      }
  return DP_OK;
}

}  // extern "C"
