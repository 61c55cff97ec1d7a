// Byte layout of the 4-bit cache's pages, shared by its append, gather and attention kernels (see the public header).
#pragma once

#include "novakv_internal.cuh"

constexpr int I4_TILE = 32;                  // tokens of a tile; a (page, KV head) chunk is two tiles
constexpr int I4_GROUP = 64;                 // channels that share a (scale, zero) pair

template <int D>
struct I4Layout {
    static constexpr int GROUPS = D / I4_GROUP;
    static constexpr int PIECES = D / 32;                          // 16-byte pieces of a token's codes
    static constexpr int ROW = D / 2;                              // code bytes of a token
    static constexpr int CODES = I4_TILE * ROW;                    // of a tile; its (scale, zero) pairs follow
    static constexpr int TILE_BYTES = CODES + I4_TILE * GROUPS * 4;
    static constexpr int CHUNK_BYTES = 2 * TILE_BYTES;
    // Piece p of row t is kept at p ^ swizzle(t): the eight rows that one shared-memory matrix load touches at a time then
    // lie in different banks (rows of 64 bytes would meet in four, rows of 32 in two).
    __host__ __device__ static constexpr int swizzle(int t) { return D == 128 ? (t >> 1) & 3 : (t >> 2) & 1; }
    // byte of channels 8 u .. 8 u + 7 (one 32-bit word) of row t in a tile
    __host__ __device__ static constexpr int word(int t, int u) { return t * ROW + (((u >> 2) ^ swizzle(t)) << 4) + ((u & 3) << 2); }
    __host__ __device__ static constexpr int pair(int t, int g) { return CODES + (t * GROUPS + g) * 4; }
};
