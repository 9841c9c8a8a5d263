// Launches of the calls around the tree attention (tree_ops.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "tree.hpp"

namespace cptree {

hipError_t launch_layout(const int32_t* parents, const NodeRows& rows, int n_rows, uint64_t* mask,
                         int words, int32_t* positions, hipStream_t s);

// The vocabulary's pieces, one workgroup each, when T nodes' logits are read.
int verify_pieces(int64_t n_tokens, int32_t vocab);
// The most candidates, nodes times pieces, of batches of up to T nodes.
int64_t verify_candidates(int64_t n_tokens, int32_t vocab);

hipError_t launch_argmax(const uint16_t* logits, int64_t ld, int32_t vocab, int64_t n_tokens,
                         int pieces, uint64_t* best, hipStream_t s);
hipError_t launch_walk(const uint64_t* best, int pieces, const int32_t* tokens,
                       const int32_t* parents, const NodeRows& rows, int n_rows, int row0,
                       int max_path, int32_t* target, int32_t* path, int32_t* n_accepted,
                       int32_t* next_token, hipStream_t s);

struct PoolArgs {
  int d, block, hkv, mbr, num_blocks, n_layers;
};

hipError_t launch_compact(const PoolArgs& a, const Layers& layers, const int32_t* bt,
                          const MoveRows& rows, int n_rows, const int32_t* path, int max_path,
                          const int32_t* n_accepted, hipStream_t s);
hipError_t launch_fork(const PoolArgs& a, const Layers& layers, int32_t* bt, const Forks& forks,
                       int n_forks, bool tables, hipStream_t s);

}  // namespace cptree
