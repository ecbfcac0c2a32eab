// A cache held in 4 bits: how a row of one head lies in memory (fc_cache4.cu writes it, fc_decode_ex.cu reads it).
//
// A row of d channels is two halves of d/2; a half has a scale and a minimum in the cache's 16-bit type, and a channel's
// value is  min + scale * code,  code 0..15.  Per head the rows are consecutive: codes [capacity][d/2] bytes, parameters
// [capacity][4] = (scale, min) of the first and of the second half.  So a tile of rows is one run of bytes per array, which
// one bulk copy brings in.  The order of the codes inside a row is the one in which a warp of the decoding kernel needs
// them as operands of m16n8k16 products, lane (g, t) = (lane / 4, lane % 4):
//   keys    the channels are the products' depth.  A lane needs, per 16 channels ("slice" s), four of its row g: channels
//           16 s + 4 t + i, i = 0..3.  Run t (d/8 bytes) of a row holds them for all s; word s/2 of the run has slice s at
//           nibbles (i & 1) * 4 + (i >> 1) + 2 * (s & 1): masks 0x000f000f and 0x00f000f0 of the word (of the word >> 8 for
//           odd slices) are then pairs (i = 0, 1) and (i = 2, 3) as 16-bit numbers.
//   values  the channels are the rows of the product.  A lane needs channels 8 n + g of all n: run g (d/16 bytes) of a row
//           has them as nibbles n = 0, 1, ...
// A code left in place in a 16-bit word is the subnormal half number code * 2^-24 (or, in the second nibble, code * 2^-20),
// exact, so a mask is all the unpacking that the tensor cores' operands need.
#pragma once
#include "fc_common.cuh"

namespace cache4 {

constexpr int kGroups = 2;                           // halves of a row
constexpr int kParamBytes = 2 * kGroups * 2;         // per row, head and matrix

__host__ __device__ constexpr int code_bytes(int d) { return d / 2; }

inline fc_status check(const fc_cache4 *c) {
  if (!c || !c->codes_k || !c->codes_v || !c->params_k || !c->params_v) return FC_ERR_INVALID_ARG;
  if (c->capacity_rows < 16 || c->capacity_rows % 16 != 0 || c->num_heads < 1) return FC_ERR_INVALID_ARG;
  if (c->dtype != FC_F16 && c->dtype != FC_BF16) return FC_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return FC_ERR_UNSUPPORTED;
  if (c->capacity_rows > 0x7fffffffll - 4096 || c->num_heads > 65535) return FC_ERR_UNSUPPORTED;
  if (((uintptr_t)c->codes_k & 15) || ((uintptr_t)c->codes_v & 15) || ((uintptr_t)c->params_k & 15) || ((uintptr_t)c->params_v & 15))
    return FC_ERR_INVALID_ARG;
  return FC_OK;
}

}  // namespace cache4
