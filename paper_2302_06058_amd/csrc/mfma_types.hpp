// Operand registers of the bf16 matrix instructions, and the plain end of a product, for the main loops in the *_body.hpp files.
#pragma once
#include "common.hpp"

namespace bimask {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(__bf16)))) __bf16 bf16x16;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));   // native 16-byte register vector
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

union BFrag { bf16x16 v; bf16x8 half[2]; u32x4 q[2]; };           // tokens: a sparse instruction's, or two dense ones'
union AFrag { bf16x8 v; u32x4 q; };                               // weights

struct PlainOut { static constexpr bool kFused = false; };        // sums are rounded and written, nothing more

}  // namespace
}  // namespace bimask
