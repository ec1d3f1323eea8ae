// A matrix in 8 bits with a power-of-two scale per 32 columns, and back.
//
// q = rint(x * 2^-e), e the least with 127 * 2^e >= max |x| of the group: the scale is a power of
// two, so neither the product nor reading back rounds (127 multiples fit the 8-bit significand of
// bf16; in f16 magnitudes past its range are read as its largest).  Both kernels are bound by the
// bytes that they move: a thread takes 8 columns (16 bytes of a 16-bit type, 8 of the packed
// values), four neighbouring lanes make a group and find its largest magnitude with two lane
// exchanges.  8192 x 10944 in bf16, packed and read back: 93 us for 549 MB,
// 5.9 TB/s (part of it out of the last-level cache).
#pragma once

#include "lm_types.hpp"

namespace lm {

template <typename T>
__global__ __launch_bounds__(256) void k_q8_pack(const T* __restrict__ x, int64_t ldx,
                                                 int64_t rows, int n, int8_t* __restrict__ q,
                                                 uint8_t* __restrict__ exps) {
  const int groups = groups_of(n);
  Piece p = piece_of((int64_t)blockIdx.x * 256, groups * 4);
  if (p.row >= rows) return;  // whole groups of lanes leave together
  float v[8];
  load_row_end<T, 8>(x + p.row * ldx + p.col, n - p.col, v);
  const int e = group_exponent4(v);
  store_global(q + p.row * groups * kGroup + p.col, pack8(v, e));
  if ((threadIdx.x & 3) == 0)
    store_global(exps + p.row * groups + p.col / kGroup, (uint8_t)e);
}

template <typename T>
__global__ __launch_bounds__(256) void k_q8_unpack(const int8_t* __restrict__ q,
                                                   const uint8_t* __restrict__ exps,
                                                   int64_t rows, int n, T* __restrict__ x,
                                                   int64_t ldx) {
  const int groups = groups_of(n);
  Piece p = piece_of((int64_t)blockIdx.x * 256, groups * 4);
  if (p.row >= rows || p.col >= n) return;
  const u32x2 w = load_global<u32x2>(q + p.row * groups * kGroup + p.col);
  float v[8];
  unpack8_as<T>(w, load_global<uint8_t>(exps + p.row * groups + p.col / kGroup), v);
  store_row<T, 8>(x + p.row * ldx + p.col, n - p.col, v);
}

}  // namespace lm
