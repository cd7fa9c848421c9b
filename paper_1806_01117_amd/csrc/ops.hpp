// Launch arguments of the operators of ambptt_ops.h (ops.hip checks them, the
// kernels live in attn.hip and norm.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "ambptt_ops.h"

namespace ambptt {

// sets ambptt_last_error()'s message of this thread and returns s (runtime.hip)
ambptt_status fail_with(ambptt_status s, const char* msg);

// A [batch][steps][heads][size] operand; strides in elements.
struct View {
  void* p;
  int64_t batch, step, head;
};

struct AttnArgs {
  int bf16, B, H, G, dk, dv;
  int64_t T;
  float scale;
  View q, k, v, o;
  const float* log_decay;
  const float* s0;
  const int32_t* lengths;
  float* sn;
  char* ws;
};

struct AttnGradArgs {
  AttnArgs a;  // o: the gradient of the output; sn unused
  const float* dsn;
  View dq, dk, dv;
  float* ds0;
};

size_t attn_workspace(const AttnArgs& a, bool backward);
hipError_t launch_attn(const AttnArgs& a, hipStream_t s);
hipError_t launch_attn_step(const AttnArgs& a, hipStream_t s);  // T = 1
hipError_t launch_attn_backward(const AttnGradArgs& a, hipStream_t s);

struct DropArgs {
  uint32_t at;  // an element is kept where its 16 bits are >= at; 0: no dropout
  float up;     // factor of what is kept
  uint64_t seed, offset;
};

struct Rows {
  void* p;
  int64_t ld;  // elements from one row to the next
};

struct DropoutArgs {
  int bf16;
  int64_t rows, cols;
  DropArgs d;
  Rows x, r, y;  // r.p NULL: none
};
hipError_t launch_dropout(const DropoutArgs& a, hipStream_t s);

struct NormArgs {
  int bf16, f8, block;
  int64_t rows;
  int cols;
  float eps;
  DropArgs d;
  Rows x, r, h, y;
  const float* w;
  float* scale;
};
hipError_t launch_add_norm(const NormArgs& a, hipStream_t s);

struct NormGradArgs {
  int bf16;
  int64_t rows;
  int cols;
  float eps;
  DropArgs d;
  Rows dy, dh, h, dr, dx;
  const float* w;
  float* dw;
  float* parts;  // [norm_grad_parts][cols]
};
int norm_grad_parts(int64_t rows, int64_t cols);
hipError_t launch_add_norm_backward(const NormGradArgs& a, hipStream_t s);

}  // namespace ambptt
