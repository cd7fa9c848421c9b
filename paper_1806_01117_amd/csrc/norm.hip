// Dropout, and the root-mean-square norm behind the residual's addition.
#include "ops.hpp"

namespace ambptt {

namespace {

constexpr int kThreads = 256;
constexpr int kV = 8;  // columns per thread and step: the elements of one counter

// Philox-4x32-10: the 128 bits of counter n under a 64-bit key.
__device__ __forceinline__ uint4 philox(uint64_t n, uint64_t key) {
  uint32_t k0 = uint32_t(key), k1 = uint32_t(key >> 32);
  uint4 x = {uint32_t(n), uint32_t(n >> 32), 0, 0};
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = uint64_t(x.x) * 0xD2511F53u, b = uint64_t(x.z) * 0xCD9E8D57u;
    x = {uint32_t(b >> 32) ^ x.y ^ k0, uint32_t(b), uint32_t(a >> 32) ^ x.w ^ k1, uint32_t(a)};
    k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
  }
  return x;
}

// dropout of the eight columns of counter n; what is dropped is zero whatever it held
__device__ __forceinline__ void drop8(float (&v)[kV], const DropArgs& d, uint64_t n) {
  const uint4 x = philox(n, d.seed);
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const uint32_t u = i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
    v[i] = u >= d.at ? v[i] * d.up : 0.0f;
  }
}

// columns c .. c + 7 of row r as fp32; zeros past the row's end
template <class T>
__device__ __forceinline__ void load8(float (&v)[kV], const Rows& x, int64_t r, int64_t c, int64_t cols) {
  const T* p = static_cast<const T*>(x.p) + r * x.ld + c;
#pragma unroll
  for (int i = 0; i < kV; ++i) v[i] = c + i < cols ? float(p[i]) : 0.0f;
}
template <class T>
__device__ __forceinline__ void store8(const float (&v)[kV], const Rows& x, int64_t r, int64_t c, int64_t cols) {
  T* p = static_cast<T*>(x.p) + r * x.ld + c;
#pragma unroll
  for (int i = 0; i < kV; ++i)
    if (c + i < cols) p[i] = T(v[i]);
}

template <class T>
__global__ __launch_bounds__(kThreads) void dropout(DropoutArgs a) {
  const int64_t wide = (a.cols + kV - 1) / kV;
  const int64_t c8 = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  if (c8 >= wide) return;
  for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
    float v[kV];
    load8<T>(v, a.x, r, c8 * kV, a.cols);
    if (a.d.at) drop8(v, a.d, a.d.offset + r * wide + c8);
    if (a.r.p) {
      float q[kV];
      load8<T>(q, a.r, r, c8 * kV, a.cols);
#pragma unroll
      for (int i = 0; i < kV; ++i) v[i] += q[i];
    }
    store8<T>(v, a.y, r, c8 * kV, a.cols);
  }
}

// the sum (or the maximum) over a workgroup, in every thread; a fixed order
template <bool MAX>
__device__ __forceinline__ float block_all(float v, float* lds) {
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    const float u = __shfl_xor(v, o);
    v = MAX ? fmaxf(v, u) : v + u;
  }
  __syncthreads();  // the last call's values are read
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int i = 1; i < kThreads / 64; ++i) v = MAX ? fmaxf(v, lds[i]) : v + lds[i];
  return v;
}

template <class T>
__device__ __forceinline__ void load_h(float (&v)[kV], const NormArgs& a, int64_t r, int64_t c, int64_t wide) {
  load8<T>(v, a.x, r, c, a.cols);
  if (a.d.at) drop8(v, a.d, a.d.offset + r * wide + c / kV);
  if (a.r.p) {
    float q[kV];
    load8<T>(q, a.r, r, c, a.cols);
#pragma unroll
    for (int i = 0; i < kV; ++i) v[i] += q[i];
  }
}

// the stored e4m3 of a pair
__device__ __forceinline__ uint32_t f8x2(float a, float b) {
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false)) & 0xffffu;
}

// One workgroup per row, which is read again for each pass over it (h may be
// x or the residual, so it is stored in the last).
template <class T>
__global__ __launch_bounds__(kThreads) void add_norm(NormArgs a) {
  __shared__ float lds[kThreads / 64];
  const int64_t wide = (a.cols + kV - 1) / kV;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    float sum = 0.0f;
    for (int64_t c = threadIdx.x * kV; c < a.cols; c += kThreads * kV) {
      float v[kV];
      load_h<T>(v, a, r, c, wide);
#pragma unroll
      for (int i = 0; i < kV; ++i) sum += v[i] * v[i];
    }
    const float rr = rsqrtf(block_all<false>(sum, lds) / float(a.cols) + a.eps);
    float most = 0.0f;
    if (a.f8 && !a.block) {
      for (int64_t c = threadIdx.x * kV; c < a.cols; c += kThreads * kV) {
        float v[kV];
        load_h<T>(v, a, r, c, wide);
#pragma unroll
        for (int i = 0; i < kV; ++i)
          if (c + i < a.cols) most = fmaxf(most, fabsf(a.w[c + i] * (v[i] * rr)));
      }
      most = block_all<true>(most, lds);
    }
    // every thread goes through the same steps: 16 lanes share a block's maximum
    for (int64_t c0 = 0; c0 < a.cols; c0 += kThreads * kV) {
      const int64_t c = c0 + threadIdx.x * kV;
      float v[kV], y[kV];
      load_h<T>(v, a, r, c, wide);
#pragma unroll
      for (int i = 0; i < kV; ++i) y[i] = c + i < a.cols ? a.w[c + i] * (v[i] * rr) : 0.0f;
      if (a.h.p) store8<T>(v, a.h, r, c, a.cols);
      if (!a.f8) {
        store8<T>(y, a.y, r, c, a.cols);
        continue;
      }
      float top = most;
      if (a.block) {
        top = 0.0f;
#pragma unroll
        for (int i = 0; i < kV; ++i) top = fmaxf(top, fabsf(y[i]));
#pragma unroll
        for (int o = 8; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
      }
      const float scale = top > 0.0f ? top / 448.0f : 1.0f;
      if (c < a.cols) {
        if (a.block ? threadIdx.x % 16 == 0 : c == 0)
          a.scale[a.block ? r * ((a.cols + 127) / 128) + c / 128 : r] = scale;
        uint8_t* p = static_cast<uint8_t*>(a.y.p) + r * a.y.ld + c;
#pragma unroll
        for (int i = 0; i < kV; i += 2) {
          const uint32_t u = f8x2(y[i] / scale, y[i + 1] / scale);
          if (c + i < a.cols) p[i] = u & 0xff;
          if (c + i + 1 < a.cols) p[i + 1] = u >> 8;
        }
      }
    }
  }
}

// Rows blockIdx.x, blockIdx.x + gridDim.x, ...: their dr, dx, and their sum of
// dy h r in the workgroup's row of parts.
template <class T>
__global__ __launch_bounds__(kThreads) void add_norm_backward(NormGradArgs a) {
  __shared__ float lds[kThreads / 64];
  const int64_t wide = (a.cols + kV - 1) / kV;
  const float inv = 1.0f / float(a.cols);
  bool first = true;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x, first = false) {
    float hh = 0.0f, ah = 0.0f;
    for (int64_t c = threadIdx.x * kV; c < a.cols; c += kThreads * kV) {
      float h[kV], dy[kV];
      load8<T>(h, a.h, r, c, a.cols);
      load8<T>(dy, a.dy, r, c, a.cols);
#pragma unroll
      for (int i = 0; i < kV; ++i)
        if (c + i < a.cols) hh += h[i] * h[i], ah += a.w[c + i] * dy[i] * h[i];
    }
    hh = block_all<false>(hh, lds), ah = block_all<false>(ah, lds);
    const float rr = rsqrtf(hh * inv + a.eps), m = rr * rr * (ah * inv);
    for (int64_t c = threadIdx.x * kV; c < a.cols; c += kThreads * kV) {
      float h[kV], dy[kV], dr[kV];
      load8<T>(h, a.h, r, c, a.cols);
      load8<T>(dy, a.dy, r, c, a.cols);
      if (a.dh.p) {
        load8<T>(dr, a.dh, r, c, a.cols);
      } else {
#pragma unroll
        for (int i = 0; i < kV; ++i) dr[i] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < kV; ++i)
        if (c + i < a.cols) {
          dr[i] += rr * (a.w[c + i] * dy[i] - h[i] * m);
          if (a.dw) {
            float* p = a.parts + int64_t(blockIdx.x) * a.cols + c + i;
            *p = (first ? 0.0f : *p) + dy[i] * (h[i] * rr);
          }
        }
      store8<T>(dr, a.dr, r, c, a.cols);
      if (a.dx.p) {
        if (a.d.at) drop8(dr, a.d, a.d.offset + r * wide + c / kV);
        store8<T>(dr, a.dx, r, c, a.cols);
      }
    }
  }
}

// dw = the sum of `parts` rows, in order
__global__ __launch_bounds__(kThreads) void sum_parts(const float* p, int parts, int cols, float* out) {
  const int64_t c = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  if (c >= cols) return;
  float v = 0.0f;
  for (int i = 0; i < parts; ++i) v += p[int64_t(i) * cols + c];
  out[c] = v;
}

unsigned blocks(int64_t n, int64_t most) { return unsigned(n < 1 ? 1 : n < most ? n : most); }

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s) {
  const int64_t wide = (a.cols + kV - 1) / kV;
  const dim3 grid(unsigned((wide + kThreads - 1) / kThreads), blocks(a.rows, 65535));
  if (a.bf16)
    dropout<__bf16><<<grid, kThreads, 0, s>>>(a);
  else
    dropout<float><<<grid, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_add_norm(const NormArgs& a, hipStream_t s) {
  const unsigned grid = blocks(a.rows, 65535);
  if (a.bf16)
    add_norm<__bf16><<<grid, kThreads, 0, s>>>(a);
  else
    add_norm<float><<<grid, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

int norm_grad_parts(int64_t rows, int64_t) { return int(blocks(rows, 512)); }

hipError_t launch_add_norm_backward(const NormGradArgs& a, hipStream_t s) {
  const unsigned parts = unsigned(norm_grad_parts(a.rows, a.cols));
  if (a.rows) {
    if (a.bf16)
      add_norm_backward<__bf16><<<parts, kThreads, 0, s>>>(a);
    else
      add_norm_backward<float><<<parts, kThreads, 0, s>>>(a);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  if (!a.dw) return hipSuccess;
  sum_parts<<<unsigned((a.cols + kThreads - 1) / kThreads), kThreads, 0, s>>>(a.parts, a.rows ? int(parts) : 0, a.cols, a.dw);
  return hipGetLastError();
}

}  // namespace ambptt
