// What the entry points of the serving forms (serving_api.cpp) and their kernels (quantize.hip, moe.hip) share.
#ifndef EMBX_SERVING_HPP
#define EMBX_SERVING_HPP

#include <cstdint>

#include "dense.hpp"

namespace embx {

// Rows of x to 8-bit integers and their scales.
struct Quantize {
  const void* x;
  int8_t* q;
  float* scale;
  int64_t ldx, ldq, m;
  int32_t k, padded;       // q's rows are written with zeros up to `padded` elements
};

// A layer of experts.  The matrices: gate, up, down.
struct Moe {
  const void* x;
  const void* router;
  const void* w[3];
  const float* scale[3];   // 8-bit matrices, or NULL
  void* h;                 // [m * top_k][ldh]: act(gate) * up of each row's experts
  void* y;
  int32_t* chosen;         // [m][top_k]
  float* share;            // [m][top_k]
  int64_t ldx, ldr, ldh, ldy, ldw[3], stride[3];
  int32_t m, f, d, experts, top_k, act, renormalize;
};

constexpr int kMostExperts = 1024, kMostTopK = 32;

int quantize_launch(int dtype, const Quantize& a, void* stream);

// launches of the kernels of one type (moe.hip is compiled once per type); 0 or a hipError_t
int moe_launch_f32(const Moe& a, void* stream);
int moe_launch_f16(const Moe& a, void* stream);
int moe_launch_bf16(const Moe& a, void* stream);

}  // namespace embx
#endif
