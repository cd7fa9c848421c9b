// Attention whose state decays: the recurrence, token by token.
//
// The forward pass and the three gradients are one recurrence on different
// operands.  A state [na][nb] takes rank-1 updates from rows u and w, and each
// row c is multiplied by it:
//   o:  u = k, w = v, c = q, forwards         S_i = l S_{i-1} + k_i v_i^T
//   dq: u = v, w = k, c = do, forwards        (S_i^T)
//   dv: u = q, w = do, c = k, backwards       A_i = D_i + scale sum q_i do_i^T
//   dk: u = do, w = q, c = v, backwards       (A_i^T), D_{i-1} = l A_i
#include "ops.hpp"

namespace ambptt {

namespace {

struct RecurArgs {
  View u, w, c, out;  // updates [B][T][H gu], products [B][T][H gc]
  int gu, gc, na, nb;
  int64_t T;
  int H;
  float up, mul;  // factors of the updates and of the products
  const float* log_decay;
  const int32_t* lengths;
  const float* s0;  // state at row r, column c: s0[r * sr + c * sc], NULL = zeros
  float* sn;        // the last state, the same layout, or NULL
  int sr, sc;
};

template <class T>
__device__ __forceinline__ float get(const View& v, int b, int64_t t, int h, int i) {
  return float(static_cast<const T*>(v.p)[b * v.batch + t * v.step + h * v.head + i]);
}

// One workgroup per state; a thread holds one column of it.
template <class T, int NA, bool BACK>
__global__ __launch_bounds__(128) void recur(RecurArgs a) {
  __shared__ float row[NA];
  const int h = blockIdx.x, b = blockIdx.y, e = threadIdx.x;
  const bool has = e < a.nb;
  // lambda - 1: fp32 holds it to 24 bits where lambda itself, rounded, would be
  // off by n 2^-25 after n tokens
  const float less = expm1f(a.log_decay[h]);
  int64_t n = a.T;
  if (a.lengths) n = min(max(int64_t(a.lengths[b]), int64_t(0)), a.T);
  const int64_t st = int64_t(b * a.H + h) * a.na * a.nb;
  float S[NA];
#pragma unroll
  for (int r = 0; r < NA; ++r) S[r] = a.s0 && has && r < a.na ? a.s0[st + r * a.sr + e * a.sc] : 0.0f;
  for (int64_t i = 0; i < n; ++i) {
    const int64_t t = BACK ? n - 1 - i : i;
    if (!BACK) {
#pragma unroll
      for (int r = 0; r < NA; ++r) S[r] = fmaf(S[r], less, S[r]);
    }
    for (int g = 0; g < a.gu; ++g) {
      __syncthreads();
      if (e < NA) row[e] = e < a.na ? get<T>(a.u, b, t, h * a.gu + g, e) : 0.0f;
      const float w = has ? a.up * get<T>(a.w, b, t, h * a.gu + g, e) : 0.0f;
      __syncthreads();
#pragma unroll
      for (int r = 0; r < NA; ++r) S[r] += row[r] * w;
    }
    for (int g = 0; g < a.gc; ++g) {
      __syncthreads();
      if (e < NA) row[e] = e < a.na ? get<T>(a.c, b, t, h * a.gc + g, e) : 0.0f;
      __syncthreads();
      float o = 0.0f;
#pragma unroll
      for (int r = 0; r < NA; ++r) o += row[r] * S[r];
      if (has) static_cast<T*>(a.out.p)[b * a.out.batch + t * a.out.step + (h * a.gc + g) * a.out.head + e] = T(a.mul * o);
    }
    if (BACK) {
#pragma unroll
      for (int r = 0; r < NA; ++r) S[r] = fmaf(S[r], less, S[r]);
    }
  }
  for (int64_t t = n; t < a.T; ++t)
    for (int g = 0; g < a.gc; ++g)
      if (has) static_cast<T*>(a.out.p)[b * a.out.batch + t * a.out.step + (h * a.gc + g) * a.out.head + e] = T(0.0f);
  if (a.sn && has) {
#pragma unroll
    for (int r = 0; r < NA; ++r)
      if (r < a.na) a.sn[st + r * a.sr + e * a.sc] = S[r];
  }
}

template <class T, int NA>
hipError_t run_recur(const RecurArgs& a, int B, bool back, hipStream_t s) {
  const dim3 grid(a.H, B);
  if (back)
    recur<T, NA, true><<<grid, 128, 0, s>>>(a);
  else
    recur<T, NA, false><<<grid, 128, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_recur(const RecurArgs& a, int bf16, int B, bool back, hipStream_t s) {
  if (bf16) return a.na <= 64 ? run_recur<__bf16, 64>(a, B, back, s) : run_recur<__bf16, 128>(a, B, back, s);
  return a.na <= 64 ? run_recur<float, 64>(a, B, back, s) : run_recur<float, 128>(a, B, back, s);
}

RecurArgs base(const AttnArgs& a) {
  RecurArgs r{};
  r.T = a.T, r.H = a.H, r.up = 1.0f, r.mul = 1.0f, r.log_decay = a.log_decay, r.lengths = a.lengths;
  return r;
}

}  // namespace

size_t attn_workspace(const AttnArgs&, bool) { return 0; }

hipError_t launch_attn(const AttnArgs& a, hipStream_t s) {
  RecurArgs r = base(a);
  r.u = a.k, r.w = a.v, r.c = a.q, r.out = a.o, r.gu = 1, r.gc = a.G, r.na = a.dk, r.nb = a.dv;
  r.mul = a.scale, r.s0 = a.s0, r.sn = a.sn, r.sr = a.dv, r.sc = 1;
  return launch_recur(r, a.bf16, a.B, false, s);
}

hipError_t launch_attn_backward(const AttnGradArgs& g, hipStream_t s) {
  const AttnArgs& a = g.a;
  RecurArgs r = base(a);
  r.u = a.v, r.w = a.k, r.c = a.o, r.out = g.dq, r.gu = 1, r.gc = a.G, r.na = a.dv, r.nb = a.dk;
  r.mul = a.scale, r.s0 = a.s0, r.sr = 1, r.sc = a.dv;
  hipError_t e = launch_recur(r, a.bf16, a.B, false, s);
  if (e != hipSuccess) return e;
  r = base(a);
  r.up = a.scale, r.s0 = g.dsn;
  r.u = a.o, r.w = a.q, r.c = a.v, r.out = g.dk, r.gu = a.G, r.gc = 1, r.na = a.dv, r.nb = a.dk, r.sr = 1, r.sc = a.dv;
  e = launch_recur(r, a.bf16, a.B, true, s);
  if (e != hipSuccess) return e;
  r.u = a.q, r.w = a.o, r.c = a.k, r.out = g.dv, r.na = a.dk, r.nb = a.dv, r.sr = a.dv, r.sc = 1, r.sn = g.ds0;
  return launch_recur(r, a.bf16, a.B, true, s);
}

}  // namespace ambptt
