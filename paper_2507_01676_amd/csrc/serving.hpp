// What the entry points of the serving forms (serving_api.cpp) and their kernels (quantize.hip, moe.hip) share.
#ifndef EMBX_SERVING_HPP
#define EMBX_SERVING_HPP

#include <cstdint>

#include "../../include/embx_serving.h"
#include "dense.hpp"

namespace embx {

// Rows of x to 8-bit integers and their scales.
struct Quantize {
  const void* x;
  int8_t* q;
  float* scale;
  int64_t ldx, ldq, m;
  int32_t k, padded;       // q's rows are written with zeros up to `padded` elements
  DensePack pack;          // 8-bit matrices that the same launch copies
  uint32_t groups;         // workgroups for the rows (set by the launch); those behind them copy
};

// Which kernels a layer of experts takes.
struct MoeChoice {
  int32_t up_variant, down_variant;   // MoeVariant
  int32_t up_blocks;       // kMoeMany: 16s of rows at a time, 2 or, of weights of 16 bits, 4
  int32_t up_waves;        // wavefronts that share a reduction of the up projections: 1, 2, 4 or 8
  int32_t up_parts;        // workgroups that share an expert's rows and columns of the up projections
  int32_t fused;           // every workgroup of the up projections routes by itself: see kFused and kPicked
  int32_t apart;           // a launch of its own works the logits out
  int32_t down_waves;      // of the down projection.  kMoeFew: wavefronts of a workgroup, 8 or 16; kMoeMany: that share a reduction
  int32_t down_parts, down_blocks;   // kMoeMany: workgroups that share an expert's rows and columns, and 16s of rows at a time
  int32_t down_rows;       // of x that a workgroup of the down projection has: kDownRows, and kUses / top_k, at most
  int32_t splits;          // workgroups that share those rows and its columns
  int32_t chunk;           // of the down projection's reduction, that a wavefront takes at a time
};

MoeChoice moe_choose(const emb_moe_t& a);

// A layer of experts.  The matrices: gate, up, down.
struct Moe : MoeChoice {
  const void* x;
  const void* router;
  const void* w[3];
  const float* scale[3];   // 8-bit matrices, or NULL
  float* h;                // [m * top_k][ldh]: act(gate) * up of each row's experts
  void* y;
  int32_t* chosen;         // [m][top_k]
  float* share;            // [m][top_k]
  int64_t ldx, ldr, ldh, ldy, ldw[3], stride[3];
  float* partial;          // [splits][m][d], with splits > 1; kMoeMany: [m][top_k][d]
  int32_t m, f, d, experts, top_k, act, renormalize;
  double* logits;          // [m][experts], which a launch of its own works out, or NULL
  int32_t whole;           // rows of all operands start at multiples of 16 bytes
};

// How many rows of x an expert has at a time: at most 4 (by 4 rows of weights), 16, or several times 16; of the down
// projection kMoeMany works by experts, the others by rows.
enum MoeVariant { kMoeFew = 0, kMoeMore = 1, kMoeMany = 2 };

// Logits of all rows that every workgroup of the up projections works out, or of which it picks the experts, by itself
constexpr int kFused = 16, kPicked = 256;

constexpr int kMostExperts = 1024, kMostTopK = 32;
constexpr int kUses = 512;       // uses, row * top_k + place, that a workgroup looks at at a time
constexpr int kDownRows = 64;

int quantize_launch(int dtype, const Quantize& a, void* stream);

// launches of the kernels of one type (moe.hip is compiled once per type); 0 or a hipError_t
int moe_launch_f32(const Moe& a, void* stream);
int moe_launch_f16(const Moe& a, void* stream);
int moe_launch_bf16(const Moe& a, void* stream);

}  // namespace embx
#endif
