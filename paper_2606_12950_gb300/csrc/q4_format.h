// q4_format.h -- blocks held in 4 bits (KV_Q4 layouts): sizes, and where each
// value lies.  Not part of the ABI.
//
// A block holds [Hkv][bs / 16] tiles of 16 tokens of one KV head, 18 d bytes
// each (d columns, NG = d / 64 groups of 64):
//     8 d    K codes
//     8 d    V codes
//     128 NG parameters, [16 tokens][K, V][NG] of (s, z) bf16 pairs, s in the
//            low half
// so that one copy of a tile brings all that a warp needs of 16 tokens, and each
// value lies where the lane that multiplies it reads it: with lane = 4 g + t (g
// in 0..7, t in 0..3),
//   K  token r, lane part t: d / 32 words at r d/2 + t d/8.  Word j holds columns
//      64 (j / 2) + 32 (j % 2) + 8 t + i, i = 0..7, column i in nibble i.  (Of
//      rows r = g and g + 8 lane (g, t) reads one 16-byte word each at d = 128.)
//   V  group of columns v, lane: four words at 512 v + 16 lane.  Word m holds
//      columns e = 64 v + 8 g + 2 m and e + 1 of tokens a = 2 t, a + 1, a + 8 and
//      a + 9, in nibbles
//          0 (a, e)       1 (a, e+1)       2 (a+8, e)   3 (a+8, e+1)
//          4 (a+1, e)     5 (a+1, e+1)     6 (a+9, e)   7 (a+9, e+1)
// A word masked with 0x000f000f (nibbles 0 and 4) is a pair of fp16 subnormals,
// codes times 2^-24 exactly, and with 0x00f000f0 (1 and 5) the same times 16:
// an operand of a matrix product costs one AND.  The factors are undone where
// they cost nothing.
#pragma once

#include <cstdint>

#include "kvpool.h"

constexpr int kQ4Tile = 16;    // tokens of a tile
constexpr int kQ4Group = 64;   // columns that share a scale
template <int D>
constexpr int kQ4TileBytes = 18 * D;

inline bool kvp_is_q4(const kv_layout &L) { return (L.head_dim & KV_Q4) != 0; }
inline int kvp_head_dim(const kv_layout &L) { return L.head_dim & ~KV_Q4; }

inline uint64_t kvp_layout_block_bytes(const kv_layout &L, int bs)
{
    const uint64_t rows = 2ull * (uint64_t)L.num_kv_heads * (uint64_t)bs, d = (uint64_t)kvp_head_dim(L);
    return kvp_is_q4(L) ? rows * d * 9 / 16 : rows * d * 2;
}
