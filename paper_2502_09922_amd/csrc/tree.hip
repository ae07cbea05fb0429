// Trees of drafted tokens: the entry points of include/ls_stage.h, the acceptance of drafts and the compaction of a
// cache to the nodes that are kept.
#include "entry.hpp"
#include "tree.hpp"

#include <algorithm>

namespace ls {

namespace {

// One wavefront to a sequence, a lane to a node.  Node i > 0 agrees if its token is what the model said behind its parent; a node
// is on if all of its path agrees; of the deepest ones on, the lowest index, the path is kept.  What the model said along
// the path are the tokens that the sequence has gained: those of the accepted drafts and one more.  Loads that wait for each other: one tree of
// 26 nodes 2.0 us, 32 of 16 3.1.
__global__ void __launch_bounds__(64)
k_tree_accept(const int32_t* __restrict__ cu, const int32_t* __restrict__ parents, const int32_t* __restrict__ tokens,
              const int32_t* __restrict__ said, int rows, int most, uint64_t* __restrict__ kept, int32_t* __restrict__ count,
              int32_t* __restrict__ emitted, int32_t* __restrict__ following) {
  const int b = blockIdx.x, lane = threadIdx.x;
  TreeSeq t{cu[b], cu[b + 1] - cu[b], 0};
  if (t.n < 0 || t.n > most || t.row0 < 0 || t.row0 > rows - t.n) t.n = 0;
  const bool in = lane < t.n;
  const int up = in && lane > 0 ? parents[t.row0 + lane] : -1;
  const int here = in ? said[t.row0 + lane] : -1;
  const bool agrees = in && (lane == 0 || (up >= 0 && up < lane && tokens[t.row0 + lane] == said[t.row0 + up]));
  const uint64_t path = tree_path(parents, t), ok = __builtin_amdgcn_ballot_w64(agrees);
  // depths are distinct enough for 6 bits, the lowest index wins among equals
  int rank = in && (path & ~ok) == 0 ? __builtin_popcountll(path) * TREE_MAX + (TREE_MAX - 1 - lane) : -1;
  for (int off = 32; off; off >>= 1) rank = max(rank, __shfl_xor(rank, off));
  const int best = rank < 0 ? 0 : TREE_MAX - 1 - rank % TREE_MAX;  // the root agrees always: rank < 0 only without nodes
  const uint64_t keep = (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(path >> 32), best) << 32 |
                        (unsigned)__builtin_amdgcn_readlane((int)(unsigned)path, best);
  const int n = __builtin_popcountll(keep);
  // lane j: the j-th node of the path; a kept lane finds its place by counting
  const int place = __builtin_popcountll(keep & ((1ull << lane) - 1));
  if (lane >= n) emitted[(size_t)b * TREE_MAX + lane] = -1;
  if (keep >> lane & 1) emitted[(size_t)b * TREE_MAX + place] = here;
  const int last = __builtin_amdgcn_readlane(here, best);
  if (lane == 0) {
    kept[b] = keep;
    count[b] = n;
    following[b] = last;
  }
}

// Rows of kept nodes move to the slots behind the context, all layers and heads, keys and values; a thread to a U-sized piece of a
// row.  The j-th kept node is node j or a later one, so in index order no row is overwritten before it has moved.  Eight rows are on their way at once; bound by
// its start and by two loads that wait for each other: 7B, one sequence, 26 nodes, 8 layers 5.0 us, 13B, 32 of 16 nodes, 4 layers (11
// MB) 8.4.
template <class U>
__global__ void __launch_bounds__(256)
k_tree_keep(const int32_t* __restrict__ cu, const int32_t* __restrict__ seq_lens, const uint64_t* __restrict__ kept, int rows, int most, int max_batch,
            int heads, int hkv, int max_seq, int pieces, U* __restrict__ kc, U* __restrict__ vc) {
  const int b = blockIdx.x;
  TreeSeq t;
  if (!tree_seq(cu, seq_lens, b, rows, most, max_seq, t)) return;
  uint64_t keep = kept[b];
  if (t.n < 64) keep &= (1ull << t.n) - 1;
  const int item = blockIdx.y * 256 + threadIdx.x;
  if (item >= 2 * heads * pieces) return;
  const int which = item / (heads * pieces), rest = item - which * heads * pieces;
  const int head = rest / pieces, piece = rest - head * pieces;  // head: layer * hkv + kv head
  U* base = (which ? vc : kc) + ((((size_t)(head / hkv) * max_batch + b) * hkv + head % hkv) * max_seq + t.ctx) * pieces + piece;
  constexpr int AT_ONCE = 8;
  int to = 0;
#pragma unroll 1
  while (keep) {
    U v[AT_ONCE] = {};
    int from[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      from[j] = keep ? __builtin_ctzll(keep) : -1;
      keep &= keep - 1;
      if (from[j] > to + j) v[j] = base[(size_t)from[j] * pieces];
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j)
      if (from[j] > to + j) base[(size_t)(to + j) * pieces] = v[j];
    to += AT_ONCE;
  }
}

// In a launch of its own: the one before reads the lengths in every workgroup.
__global__ void __launch_bounds__(256)
k_tree_lens(const int32_t* __restrict__ cu, const uint64_t* __restrict__ kept, int rows, int most, int max_seq, int batch, int32_t* __restrict__ seq_lens) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  TreeSeq t;
  if (b >= batch || !tree_seq(cu, seq_lens, b, rows, most, max_seq, t)) return;
  const uint64_t keep = t.n < 64 ? kept[b] & ((1ull << t.n) - 1) : kept[b];
  seq_lens[b] = t.ctx + __builtin_popcountll(keep);
}

}  // namespace

const char* heads_error(const ls_heads* h) {
  if (!h) return "NULL ls_heads";
  if (h->dtype > LS_DTYPE_BF16) return "unknown dtype";
  if (!h->n_q_heads || !h->n_kv_heads || h->n_q_heads % h->n_kv_heads || h->n_q_heads > 65535) return "n_kv_heads has to divide n_q_heads (65535 at most)";
  if (!h->head_dim || (h->head_dim & 1) || h->head_dim > 256) return "head_dim has to be even and 256 at most";
  if (!h->max_batch || !h->max_seq || h->max_seq > (1u << 24) || h->max_batch >= (1u << 24)) return "max_batch outside [1, 2^24) or max_seq outside [1, 2^24]";
  return nullptr;
}

const char* tree_error(const ls_tree* t, int batch, int max_batch, bool with_parents, int* rows, int* min_nodes, int* max_nodes) {
  if (!t || !t->cu_nodes || !t->cu_nodes_host) return "NULL ls_tree or pointer inside it";
  if (batch < 1 || batch > max_batch) return "batch outside [1, max_batch]";
  if (t->cu_nodes_host[0] != 0) return "cu_nodes has to start at 0";
  int least = LS_TREE_MAX, most = 0;
  for (int b = 0; b < batch; ++b) {
    const long n = (long)t->cu_nodes_host[b + 1] - t->cu_nodes_host[b];
    if (n < 0 || n > LS_TREE_MAX) return "a tree has 0 to 64 nodes";
    if (n > most) most = (int)n;
    if (n && n < least) least = (int)n;
  }
  *rows = t->cu_nodes_host[batch];
  *min_nodes = least;
  *max_nodes = most;
  if (with_parents && *rows && !t->parents) return "NULL parents";
  return nullptr;
}

}  // namespace ls

namespace {

using ls::bad;
using ls::launched;

}  // namespace

extern "C" {

size_t ls_tree_attention_scratch_bytes(const ls_heads* h, const ls_tree* tree, int batch, int max_ctx) {
  ls::TreeAttn a;
  int min_nodes = 0;
  if (ls::heads_error(h) || ls::tree_error(tree, batch, (int)h->max_batch, false, &a.rows, &min_nodes, &a.max_nodes)) return 0;
  if (max_ctx < 0 || a.rows == 0 || (long)max_ctx + min_nodes > (long)h->max_seq) return 0;
  a.batch = batch; a.max_keys = std::min(max_ctx + a.max_nodes, (int)h->max_seq);
  a.hq = (int)h->n_q_heads; a.hkv = (int)h->n_kv_heads; a.hd = (int)h->head_dim; a.max_seq = (int)h->max_seq;
  return ls::tree_attn_scratch_bytes(a);
}

ls_status ls_tree_attention(const ls_heads* h, const ls_tree* tree, int batch, int max_ctx, const void* qkv, const float* rope, const ls_kv* layer,
                            void* out, void* scratch, size_t scratch_bytes, void* hip_stream) {
  static const char* who = "ls_tree_attention";
  if (const char* e = ls::heads_error(h)) return bad(who, e);
  int rows = 0, min_nodes = 0, max_nodes = 0;
  if (const char* e = ls::tree_error(tree, batch, (int)h->max_batch, true, &rows, &min_nodes, &max_nodes)) return bad(who, e);
  if ((rows && (!qkv || !out)) || !layer || !layer->k || !layer->v || !layer->seq_lens) return bad(who, "NULL argument");
  const uintptr_t size = h->dtype == LS_DTYPE_F32 ? 4 : 2;
  if (((uintptr_t)qkv | (uintptr_t)out | (uintptr_t)layer->k | (uintptr_t)layer->v) & (size - 1)) return bad(who, "a buffer is not aligned to its type");
  if ((uintptr_t)rope & 7) return bad(who, "rope is not aligned to 8 bytes");
  if (max_ctx < 0) return bad(who, "max_ctx is negative");
  if (rows == 0) return LS_OK;
  if ((long)max_ctx + min_nodes > (long)h->max_seq) {
    ls::set_last_error("%s: context %d + %d nodes exceed max_seq %u", who, max_ctx, min_nodes, h->max_seq);
    return LS_ERR_KV_OVERFLOW;
  }
  ls::TreeAttn a;
  a.qkv = qkv; a.cs = rope; a.parents = tree->parents; a.cu = tree->cu_nodes; a.seq_lens = layer->seq_lens;
  a.batch = batch; a.rows = rows; a.max_nodes = max_nodes; a.max_keys = std::min(max_ctx + max_nodes, (int)h->max_seq);
  a.hq = (int)h->n_q_heads; a.hkv = (int)h->n_kv_heads; a.hd = (int)h->head_dim; a.max_seq = (int)h->max_seq;
  a.kc = layer->k; a.vc = layer->v; a.out = out;
  a.scratch = ((uintptr_t)scratch & 15) ? nullptr : (float*)scratch; a.scratch_bytes = scratch_bytes;
  ls::launch_tree_attn(h->dtype, a, (hipStream_t)hip_stream);
  return launched(who);
}

ls_status ls_tree_accept(const ls_tree* tree, int batch, const int32_t* tokens, const int32_t* said, uint64_t* kept, int32_t* count,
                         int32_t* emitted, int32_t* following, void* hip_stream) {
  static const char* who = "ls_tree_accept";
  int rows = 0, min_nodes = 0, max_nodes = 0;
  if (const char* e = ls::tree_error(tree, batch, (1 << 24) - 1, true, &rows, &min_nodes, &max_nodes)) return bad(who, e);
  if ((rows && (!tokens || !said)) || !kept || !count || !emitted || !following) return bad(who, "NULL argument");
  if ((uintptr_t)kept & 7) return bad(who, "kept is not aligned to 8 bytes");
  ls::k_tree_accept<<<batch, 64, 0, (hipStream_t)hip_stream>>>(tree->cu_nodes, tree->parents, tokens, said, rows, max_nodes, kept, count, emitted, following);
  return launched(who);
}

ls_status ls_tree_keep(const ls_heads* h, int layers, const ls_tree* tree, int batch, const uint64_t* kept, const ls_kv* kv, void* hip_stream) {
  static const char* who = "ls_tree_keep";
  if (const char* e = ls::heads_error(h)) return bad(who, e);
  int rows = 0, min_nodes = 0, max_nodes = 0;
  if (const char* e = ls::tree_error(tree, batch, (int)h->max_batch, false, &rows, &min_nodes, &max_nodes)) return bad(who, e);
  if (!kept || !kv || !kv->k || !kv->v || !kv->seq_lens) return bad(who, "NULL argument");
  if ((uintptr_t)kept & 7) return bad(who, "kept is not aligned to 8 bytes");
  if (((uintptr_t)kv->k | (uintptr_t)kv->v) & 3) return bad(who, "a cache is not aligned to 4 bytes");
  const size_t row = (size_t)h->head_dim * (h->dtype == LS_DTYPE_F32 ? 4 : 2);
  const bool wide = row % 16 == 0 && (((uintptr_t)kv->k | (uintptr_t)kv->v) & 15) == 0;
  const int pieces = (int)(row / (wide ? 16 : 4));
  if (layers < 1 || (long)layers * h->n_kv_heads * 2 * pieces > 256l * 65535) return bad(who, "layers outside [1, what a launch takes]");
  if (rows == 0) return LS_OK;
  hipStream_t st = (hipStream_t)hip_stream;
  const int heads = layers * (int)h->n_kv_heads;
  const dim3 grid(batch, (2 * heads * pieces + 255) / 256);
  if (max_nodes > 1) {  // a root alone lies where it has to
    if (wide)
      ls::k_tree_keep<ls::u32x4><<<grid, 256, 0, st>>>(tree->cu_nodes, kv->seq_lens, kept, rows, max_nodes, (int)h->max_batch, heads, (int)h->n_kv_heads,
                                                   (int)h->max_seq, pieces, (ls::u32x4*)kv->k, (ls::u32x4*)kv->v);
    else
      ls::k_tree_keep<uint32_t><<<grid, 256, 0, st>>>(tree->cu_nodes, kv->seq_lens, kept, rows, max_nodes, (int)h->max_batch, heads, (int)h->n_kv_heads,
                                                      (int)h->max_seq, pieces, (uint32_t*)kv->k, (uint32_t*)kv->v);
  }
  ls::k_tree_lens<<<(batch + 255) / 256, 256, 0, st>>>(tree->cu_nodes, kept, rows, max_nodes, (int)h->max_seq, batch, kv->seq_lens);
  return launched(who);
}

}  // extern "C"
