// Rows of a matrix to 8-bit integers with a scale each.  See include/embx_serving.h for the formulas.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/embx_serving.h"
#include "dense_device.hpp"
#include "quantize_device.hpp"
#include "serving.hpp"

namespace embx {
namespace {

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));

// Eight consecutive elements as their bits.
template <int TYPE> struct Eight { using V = u16x8; };
template <> struct Eight<kDenseF32> { using V = u32x8; };

template <int TYPE>
__device__ inline float value(uint32_t bits) {
  if constexpr (TYPE == kDenseF32) return __uint_as_float(bits);
  else if constexpr (TYPE == kDenseBF16) return __uint_as_float(bits << 16);
  else return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(bits)));
}

// of LANES threads of a workgroup of 256
template <int LANES>
__device__ inline uint32_t most_of(uint32_t v) {
  for (int step = (LANES < 64 ? LANES : 64) / 2; step > 0; step >>= 1)
    v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), step)));
  if constexpr (LANES == 256) {
    __shared__ uint32_t most[4];
    __syncthreads();   // (the last row's are read)
    if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = v;
    __syncthreads();
    v = max(max(most[0], most[1]), max(most[2], most[3]));
  }
  return v;
}

// whether this workgroup copies instead
__device__ inline bool copies(const Quantize& a) {
  if (blockIdx.x < a.groups) return false;
  const uint32_t id = blockIdx.x - a.groups;
  pack_eights(a.pack, id / a.pack.groups, id % a.pack.groups);
  return true;
}

// A row in the registers of LANES threads, CH chunks of eight elements each: read once, 16 bytes at a time, and bound by
// memory: bf16 65536 x 12800 537 us, 4.7 TB/s of both, where a copy reaches 5.0.  x's rows start at multiples of 16 bytes
// (WHOLE) or anywhere, q's at multiples of 8.
template <int TYPE, int LANES, int CH, bool WHOLE>
__global__ __launch_bounds__(256) void quantize_held(Quantize a) {
  using V = typename Eight<TYPE>::V;
  using T = typename Elem<TYPE>::T;
  constexpr int kRows = 256 / LANES;
  constexpr uint32_t kSign = TYPE == kDenseF32 ? 0x7fffffffu : 0x7fffu;
  if (copies(a)) return;
  const int lane = threadIdx.x % LANES;
  const int chunks = (a.k + 7) / 8, wide = (a.padded + 7) / 8;
  for (int64_t i = int64_t(blockIdx.x) * kRows + threadIdx.x / LANES; i < a.m; i += int64_t(a.groups) * kRows) {
    const char* const x = static_cast<const char*>(a.x) + i * a.ldx * (TYPE == kDenseF32 ? 4 : 2);
    V v[CH], most = {};
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = min(lane + c * LANES, chunks - 1) * 8;
      if constexpr (!WHOLE) {
        if (at + 8 <= a.k) {
          __builtin_memcpy(&v[c], x + at * int64_t(sizeof(T)), sizeof(V));
        } else {
          using Bits = std::conditional_t<TYPE == kDenseF32, uint32_t, uint16_t>;
#pragma unroll
          for (int e = 0; e < 8; ++e) v[c][e] = reinterpret_cast<const Bits*>(x)[min(at + e, a.k - 1)];
        }
      } else if constexpr (TYPE == kDenseF32) {   // (16 bytes with none of the row's elements are not read)
        __builtin_memcpy(&v[c], __builtin_assume_aligned(x + at * int64_t(4), 16), 16);
        __builtin_memcpy(reinterpret_cast<char*>(&v[c]) + 16, __builtin_assume_aligned(x + min(at + 4, (a.k - 1) / 4 * 4) * int64_t(4), 16), 16);
      } else {
        v[c] = *reinterpret_cast<const V*>(x + at * int64_t(2));
      }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = lane + c * LANES;
      if (at >= chunks - 1) {   // what is behind the row's end counts as zeros
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (at * 8 + e >= a.k) v[c][e] = 0;
      }
      most = __builtin_elementwise_max(most, v[c] & static_cast<decltype(most[0] + 0)>(kSign));
    }
    uint32_t largest = most[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) largest = max(largest, static_cast<uint32_t>(most[e]));
    const Scale s = Scale::of(value<TYPE>(most_of<LANES>(largest)));
    if (lane == 0) a.scale[i] = s.stored();
    int8_t* const q = a.q + i * a.ldq;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      const int at = lane + c * LANES;
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = value<TYPE>(v[c][e]);
      uint32_t out[2];
      quantize8(s, x, out);
      if (at * 8 + 8 <= a.padded) {
        *reinterpret_cast<u32x2*>(q + at * 8) = u32x2{out[0], out[1]};
      } else if (at < wide) {
        for (int e = 0; e < a.padded - at * 8; ++e) q[at * 8 + e] = static_cast<int8_t>(out[e >> 2] >> 8 * (e & 3));
      }
    }
  }
}

// Rows that are too long for that, or go to a q whose rows start anywhere: read twice, consecutive elements by consecutive
// threads.  bf16 16384 x 32768 492 us, f32 764, 3.3 and 3.5 TB/s of what has to be read and written once; bf16 65536 x 4096 to
// rows of 4097 250 us, to whole ones, in registers, 155.
template <int TYPE, int LANES>
__global__ __launch_bounds__(256) void quantize_any(Quantize a) {
  using T = typename Elem<TYPE>::T;
  constexpr int kRows = 256 / LANES, kMany = 8;   // elements of a thread under way
  if (copies(a)) return;
  const int lane = threadIdx.x % LANES;
  for (int64_t i = int64_t(blockIdx.x) * kRows + threadIdx.x / LANES; i < a.m; i += int64_t(a.groups) * kRows) {
    const T* const x = static_cast<const T*>(a.x) + i * a.ldx;
    uint32_t largest = 0;
    for (int j = lane; j < a.k; j += LANES * kMany) {
      T v[kMany];
#pragma unroll
      for (int e = 0; e < kMany; ++e) v[e] = x[min(j + e * LANES, a.k - 1)];
#pragma unroll
      for (int e = 0; e < kMany; ++e) largest = max(largest, __float_as_uint(float(v[e])) & 0x7fffffffu);
    }
    const Scale s = Scale::of(__uint_as_float(most_of<LANES>(largest)));
    if (lane == 0) a.scale[i] = s.stored();
    int8_t* const q = a.q + i * a.ldq;
    for (int j = lane; j < a.padded; j += LANES * kMany) {
      T v[kMany];
#pragma unroll
      for (int e = 0; e < kMany; ++e) v[e] = x[min(j + e * LANES, a.k - 1)];
#pragma unroll
      for (int e = 0; e < kMany; ++e)
        if (j + e * LANES < a.padded)
          q[j + e * LANES] = j + e * LANES < a.k && s.fine ? static_cast<int8_t>(s.mend(float(v[e]))) : int8_t(0);
    }
  }
}

// grid of a launch with rows of LANES threads
template <int LANES>
uint32_t grid_of(Quantize& a) {
  a.groups = static_cast<uint32_t>(std::min<int64_t>((a.m + 256 / LANES - 1) / (256 / LANES), 1 << 20));
  return a.groups + a.pack.count * a.pack.groups;
}

template <int TYPE, int LANES, int CH>
int held(Quantize a, hipStream_t s) {
  constexpr int kSize = TYPE == kDenseF32 ? 4 : 2;
  const uint32_t grid = grid_of<LANES>(a);
  if (reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && a.ldx * kSize % 16 == 0) quantize_held<TYPE, LANES, CH, true><<<grid, 256, 0, s>>>(a);
  else quantize_held<TYPE, LANES, CH, false><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

template <int TYPE, int LANES>
int any(Quantize a, hipStream_t s) {
  const uint32_t grid = grid_of<LANES>(a);
  quantize_any<TYPE, LANES><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

template <int TYPE>
int launch(const Quantize& a, hipStream_t s) {
  const bool eights = reinterpret_cast<uintptr_t>(a.q) % 8 == 0 && a.ldq % 8 == 0;
  const int chunks = (std::max(a.k, a.padded) + 7) / 8;
  if (!eights || chunks > 2048) return a.k <= 128 ? any<TYPE, 16>(a, s) : a.k <= 2048 ? any<TYPE, 64>(a, s) : any<TYPE, 256>(a, s);
  // (two chunks a lane: bf16 65536 x 512 21.7 us, one 26.6; a wavefront a row where there are many: bf16 65536 x 2048 72 us, a
  // workgroup 96, but of 1024 rows 5.2 and 4.2)
  if (chunks <= 8) return held<TYPE, 8, 1>(a, s);
  if (chunks <= 16) return held<TYPE, 8, 2>(a, s);
  if (chunks <= 32) return held<TYPE, 16, 2>(a, s);
  if (chunks <= 64) return held<TYPE, 32, 2>(a, s);
  if (chunks <= 128) return held<TYPE, 64, 2>(a, s);
  if (chunks <= 256) return a.m >= 8192 ? held<TYPE, 64, 4>(a, s) : held<TYPE, 256, 1>(a, s);
  if (chunks <= 512) return held<TYPE, 256, 2>(a, s);
  if (chunks <= 1024) return held<TYPE, 256, 4>(a, s);
  return held<TYPE, 256, 8>(a, s);
}

}  // namespace

int quantize_launch(int dtype, const Quantize& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (dtype == EMB_DTYPE_F32) return launch<kDenseF32>(a, s);
  return dtype == EMB_DTYPE_F16 ? launch<kDenseF16>(a, s) : launch<kDenseBF16>(a, s);
}

}  // namespace embx
