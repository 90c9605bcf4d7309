// The paged cache in 4-bit groups of 64 along the head (matq_paged_kv4): where things stand.
//
// 16 keys of a page make a tile of 18 head_dim bytes, keys first and then values, each as
//   codes   [head_dim / 32][16 keys][16 bytes]   element e of 32 in bits 4 (e % 2) of byte e / 2
//   groups  [head_dim / 64][16 keys][scale, low] two bf16
// so that ldmatrix reads the codes of a tile from consecutive addresses (in rows of head_dim / 2 bytes the eight rows of a matrix would fall on one or two
// groups of banks), and one bulk copy brings all that a page holds of a head.
#pragma once

#include "group4.cuh"

namespace matq {
namespace kv4 {

constexpr int kTileKeys = 16, kGroup = 64;
__host__ __device__ constexpr int tile_bytes(int D) { return 18 * D; }
__host__ __device__ constexpr int half_bytes(int D) { return 9 * D; }        // keys, or values, of a tile
__host__ __device__ constexpr int groups_at(int D) { return 8 * D; }         // behind the codes of a half

}  // namespace kv4
}  // namespace matq
