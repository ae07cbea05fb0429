// What the kernels of drafted-token trees share: limits, and a wavefront's view of one sequence's tree.
#pragma once
#include "kernels.hpp"
#include "device_util.hpp"

namespace ls {

// Chunks of the keys that workgroups of their own take, and where they leave their results.
struct TreeChunks {
  int n = 1, keys = 0;   // keys of a chunk: a multiple of 64
  float* o = nullptr;    // [chunk][row * hq + head][head_dim], not normalised
  float2* ml = nullptr;  // [chunk][row * hq + head]: maximum in score units, sum
};
void launch_tree_attn_mfma(uint32_t dt, const TreeAttn& a, const TreeChunks& p, hipStream_t st);  // head_dim 64 and 128, rows on 16 bytes

constexpr int TREE_MAX = 64;  // LS_TREE_MAX: a node for each lane, a bit of a 64-bit mask for each node

struct TreeSeq {
  int row0, n, ctx;  // rows [row0, row0 + n) of the call, cached positions
};

// The tree of sequence b.  False for one that does not take part: no nodes, no room for them behind its cached positions, or
// bounds on the device that the call was not made for (`rows` in all, `most` of a tree: TREE_MAX at most), which count as none.
__device__ __forceinline__ bool tree_seq(const int32_t* __restrict__ cu, const int32_t* __restrict__ seq_lens, int b, int rows, int most,
                                         int max_seq, TreeSeq& t) {
  t.row0 = cu[b];
  t.n = cu[b + 1] - t.row0;
  t.ctx = seq_lens[b];
  if (t.n < 0 || t.n > most || t.row0 < 0 || t.row0 > rows - t.n) t.n = 0;
  return t.n > 0 && t.ctx >= 0 && t.ctx <= max_seq - t.n;
}

// Lane i: the nodes on the path from the root to node i, itself included, as bits; 0 for lanes without a node.  A parent that
// is not in front of its child counts as none.  Paths double in length from round to round: six rounds at most, two or three
// for the trees of a few levels that drafting programs make.
__device__ __forceinline__ uint64_t tree_path(const int32_t* __restrict__ parents, const TreeSeq& t) {
  const int lane = threadIdx.x & 63;
  int up = -1;
  if (lane < t.n && lane > 0) up = parents[t.row0 + lane];
  if (up >= lane) up = -1;
  uint64_t path = lane < t.n ? 1ull << lane : 0;
  while (__builtin_amdgcn_ballot_w64(up >= 0)) {
    const int from = up < 0 ? lane : up;
    const unsigned lo = (unsigned)__shfl((int)(unsigned)path, from), hi = (unsigned)__shfl((int)(unsigned)(path >> 32), from);
    path |= (uint64_t)hi << 32 | lo;
    const int next = __shfl(up, from);
    up = up < 0 ? -1 : next;
  }
  return path;
}

}  // namespace ls
