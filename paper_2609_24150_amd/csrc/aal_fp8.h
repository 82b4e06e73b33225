// Host-side interfaces of the 8-bit operators: quantisation and the product of
// operands with a scale for each block of 128.
#pragma once

#include "aal_internal.h"

namespace aal {

constexpr int kFp8Block = 128;
enum class Fp8 : int { kE4M3 = 0, kE5M2 = 1 };
enum class Scale : int { kF32 = 0, kE8M0 = 1 };

struct QuantizeArgs {
  DType in;
  const void* x;
  int64_t rows, cols, ld;
  Fp8 format;
  Scale st;
  int block_rows;   // 1 or 128
  uint8_t* q;       // may be null, with its scale
  int64_t ld_q;
  void* scale;
  uint8_t* qt;      // may be null, with its scale
  int64_t ld_qt;
  void* scale_t;
  hipStream_t stream;
};

hipError_t launch_quantize(const QuantizeArgs& a);

struct Operand {
  const uint8_t* v;
  const void* s;
  int64_t ld, s_row, s_block;
  int format;       // Fp8
  int block_rows;   // 1 or 128
};

struct MatmulArgs {
  Operand a, b;
  Scale st;
  int64_t M, N, K;
  void* c;
  DType out;
  void* ws;
  hipStream_t stream;
};

size_t matmul_workspace_bytes(int64_t M, int64_t N, int64_t K);
hipError_t launch_matmul(const MatmulArgs& a);

}  // namespace aal
