// ops_dev.hpp -- element types of the operators' arrays: loads widened to the type they are
// computed in, stores rounded once to nearest even.
#pragma once
#include <type_traits>

#include "devmath.hpp"
#include "ops.hpp"
#include "params.hpp"

namespace bsim {
namespace {

struct F64 { typedef double T; typedef double W; };
struct F32 { typedef float T; typedef float W; };
struct BF16 { typedef __bf16 T; typedef float W; };
struct F16 { typedef _Float16 T; typedef float W; };

// f = 1 / (1 + e^-g) and r = 1 - f, each to its own relative accuracy: with e = e^-|g| the
// larger of the two is 1 / (1 + e) and the smaller one e times that.
__device__ __forceinline__ void sigmoid_pair(float g, float& f, float& r) {
  const float e = __builtin_amdgcn_exp2f(fabsf(g) * -1.4426950408889634f);
  const float big = __builtin_amdgcn_rcpf(1.0f + e), small = e * big;
  f = g < 0.0f ? small : big;
  r = g < 0.0f ? big : small;
}
__device__ __forceinline__ void sigmoid_pair(double g, double& f, double& r) {
  const double e = exp(-fabs(g)), big = 1.0 / (1.0 + e), small = e * big;
  f = g < 0.0 ? small : big;
  r = g < 0.0 ? big : small;
}

// an index or action of any of the three integer types
__device__ __forceinline__ int64_t load_int(const void* p, int type, int64_t i) {
  if (type == SIM_IT_U8) return static_cast<const uint8_t*>(p)[i];
  if (type == SIM_IT_I32) return static_cast<const int32_t*>(p)[i];
  return static_cast<const int64_t*>(p)[i];
}

// A value that the compiler finds again in each round of a loop: it would otherwise keep a pointer of its
// own for every access that depends on it and step them all from round to round, more registers than there
// are. The first is the same in all lanes of a wave.
__device__ __forceinline__ void fresh(int64_t& uniform) { asm volatile("" : "+s"(uniform)); }
__device__ __forceinline__ void fresh(int& v) { asm volatile("" : "+v"(v)); }

// A value in registers that the compiler no longer knows, so that what was computed from it before is not
// held for a later use.
template <class V>
__device__ __forceinline__ void hide(V& v) {
  if constexpr (sizeof(V) == 8 || sizeof(V) == 16 || sizeof(V) == 32) {
    typedef uint32_t Words __attribute__((ext_vector_type(sizeof(V) / 4)));
    Words w = __builtin_bit_cast(Words, v);
    asm volatile("" : "+v"(w));
    v = __builtin_bit_cast(V, w);
  }
}

// f(true) or f(false), so that the usual case is compiled without its conditions
template <class F>
__device__ __forceinline__ void either(bool c, F f) {
  if (c) f(std::true_type{});
  else f(std::false_type{});
}

}  // namespace
}  // namespace bsim
