// Where things lie in a cache of 4 bits (amap_packed).
//
// A page of a head is a run of cells of 16 tokens, a cell is one piece of memory: what attention reads of 16 tokens comes with
// one copy, codes and the groups' numbers, K and V.  Inside, the codes lie as the matrix instructions' operands want them
// in registers, so that a warp's loads from shared memory are whole and unpacking is five operations for eight codes:
//   K codes   per 32 elements ("slab") 16 tokens x 4 words; word t holds elements 8t .. 8t+7, in its o-th half the elements
//             2i + o.  Up to four slabs side by side: [token][t][slab]
//   V codes   per slab 32 lanes x 8 bytes, lane 4g + t: elements 4g .. 4g+3 of the tokens 2t, 2t+1, 2t+8, 2t+9, 16 bits a
//             token.  Up to two slabs side by side: [lane][slab]
//   numbers   per group and token K's word and V's; a word is step (low 16 bits) and low (high), both bf16
// The i-th four bits of 16 lie in the bits 4i + kTurn .. of them, the last ones' upper three in bits 0 .. 2.
// A token's bytes are its own: tokens of one cell are written independently.
#pragma once
#include <cstdint>

#include "amap_serve.h"

#ifdef __CUDACC__
#define AMAP_HD __host__ __device__ __forceinline__
#else
#define AMAP_HD inline
#endif

namespace amap_serve {

constexpr int kCell = 16;  // tokens
constexpr int kSlab = 32;  // elements

// bytes of a cell of heads of 32 `slabs` elements in `groups` groups
AMAP_HD constexpr int cell_bytes(int slabs, int groups) { return slabs * 512 + groups * 128; }

// offset of the word with elements 8c .. 8c+7 of K of token `token` of a cell
AMAP_HD int k_word_at(int slabs, int token, int c) {
  const int slab = c >> 2, first = slab & ~3, wide = slabs - first < 4 ? slabs - first : 4;
  return first * 256 + (token * 4 + (c & 3)) * 4 * wide + (slab - first) * 4;
}
// offset of the 16 bits with elements 4f .. 4f+3 of V
AMAP_HD int v_half_at(int slabs, int token, int f) {
  const int slab = f >> 3, first = slab & ~1, wide = slabs - first < 2 ? slabs - first : 2;
  return slabs * 256 + first * 256 + ((f & 7) * 4 + ((token & 7) >> 1)) * 8 * wide + (slab - first) * 8 + (token >> 3) * 4 + (token & 1) * 2;
}
// offset of K's word of numbers of a group; V's lies behind it
AMAP_HD int numbers_at(int slabs, int token, int group) { return slabs * 512 + group * 128 + token * 8; }

// Both halves of a word turned by kTurn bits: as they lie in a cell, from the i-th four bits in 4i ...  kTurn is 3 so that two
// of four, and with the half's bytes exchanged the other two, lie in the bits 3 .. 6 and 7 .. 10, which as fp16 numbers are
// code x 2^-21 and code x 2^-17, as near to the upper end of what fp16 counts evenly as they can be (serve_attend_packed.cu says why).
constexpr int kTurn = 3;
AMAP_HD constexpr uint32_t turn_halves(uint32_t w) { return (w << kTurn & 0xFFF8FFF8u) | (w >> (16 - kTurn) & 0x00070007u); }

// Checks of a description that every operator on it makes; AMAP_OK, or the refusal.
int check_packed(const amap_packed &c);

}  // namespace amap_serve
