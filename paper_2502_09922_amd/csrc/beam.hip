// Beam search beside a stage: the k best continuations of each request's beams, and the caches' reordering behind them.
#include "entry.hpp"
#include "device_util.hpp"

namespace ls {

namespace {

constexpr int BEAMS_MAX = LS_BEAMS_MAX;

// A candidate: its score in 64 bits, its place beam * vocab + token in its request.
struct Cand {
  double s;
  long at;
};
__device__ __forceinline__ bool before(Cand a, Cand b) { return a.s > b.s || (a.s == b.s && a.at < b.at); }
__device__ __forceinline__ Cand better(Cand a, Cand b) { return before(a, b) ? a : b; }
__device__ __forceinline__ Cand cand_xor(Cand c, int off) {
  Cand o;
  o.s = __shfl_xor(c.s, off);
  o.at = __shfl_xor(c.at, off);
  return o;
}

// One workgroup to a request: the rows' log-sums, then the best candidate behind the last one, k times.
__global__ void __launch_bounds__(1024)
k_beam_select(const float* __restrict__ logits, const float* __restrict__ scores, const int32_t* __restrict__ ended, int beams, int vocab, int k,
              int eos, int32_t* __restrict__ rows_out, int32_t* __restrict__ tokens, float* __restrict__ scores_out) {
  constexpr int NT = 1024, NW = NT / 64;
  __shared__ double part[NW], base[BEAMS_MAX];
  __shared__ float top[NW], most[BEAMS_MAX];
  __shared__ Cand best[NW];
  const int g = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int b = 0; b < beams; ++b) {
    const float* x = logits + ((size_t)g * beams + b) * vocab;
    float m = -INFINITY;
    for (int i = threadIdx.x; i < vocab; i += NT) m = fmaxf(m, x[i]);
    m = exchange<32, 1>(m, Max{});
    if (lane == 0) top[wave] = m;
    __syncthreads();
    for (int w = 0; w < NW; ++w) m = fmaxf(m, top[w]);
    double s = 0.;
    for (int i = threadIdx.x; i < vocab; i += NT) s += (double)__expf(x[i] - m);
    for (int off = 32; off; off >>= 1) s += __shfl_xor(s, off);
    if (lane == 0) part[wave] = s;
    __syncthreads();
    s = 0.;
    for (int w = 0; w < NW; ++w) s += part[w];
    if (threadIdx.x == 0) {  // the largest logit apart: next to a large one the rest would be lost
      base[b] = (double)scores[g * beams + b] - log(s);
      most[b] = m;
    }
    __syncthreads();
  }
  Cand last{INFINITY, -1};
  for (int j = 0; j < k; ++j) {
    Cand mine{-INFINITY, (long)beams * vocab};
    for (int b = 0; b < beams; ++b) {
      const float* x = logits + ((size_t)g * beams + b) * vocab;
      const bool end = ended && ended[g * beams + b];
      for (int i = threadIdx.x; i < vocab; i += NT) {
        Cand c{end ? (i == eos ? (double)scores[g * beams + b] : -INFINITY) : ((double)x[i] - (double)most[b]) + base[b], (long)b * vocab + i};
        if (!(c.s == c.s)) c.s = -INFINITY;
        if (before(last, c)) mine = better(mine, c);
      }
    }
    for (int off = 32; off; off >>= 1) mine = better(mine, cand_xor(mine, off));
    if (lane == 0) best[wave] = mine;
    __syncthreads();
    for (int w = 0; w < NW; ++w) mine = better(mine, best[w]);
    last = mine;
    if (threadIdx.x == 0) {
      const size_t to = (size_t)g * k + j;
      rows_out[to] = g * beams + (int)(last.at / vocab);
      tokens[to] = (int)(last.at % vocab);
      scores_out[to] = (float)last.s;
    }
    __syncthreads();
  }
}

// Sequence src[b], if it is of b's group, else b itself.
__device__ __forceinline__ int source(const int32_t* __restrict__ src, int b, int lo, int group) {
  const int s = src[b];
  return s >= lo && s < lo + group ? s : b;
}

// The positions of a request's W sequences, W or fewer, in place: a thread has a U-sized piece of all of them in registers before
// it writes any.
template <int W, class U>
__global__ void __launch_bounds__(256, 1)
k_reorder(const int32_t* __restrict__ src, const int32_t* __restrict__ first, const int32_t* __restrict__ seq_lens, int group, int max_batch, int hkv,
          int max_seq, int pieces, U* __restrict__ kc, U* __restrict__ vc) {
  const int lo = blockIdx.z * group, layer = blockIdx.y / hkv, kh = blockIdx.y % hkv;
  const int pos = (int)((blockIdx.x * 256u + threadIdx.x) / (unsigned)pieces);
  const size_t piece = blockIdx.x * 256u + threadIdx.x;
  const size_t seq = (size_t)hkv * max_seq * pieces;
  const size_t at = ((size_t)layer * max_batch * hkv + kh) * max_seq * pieces + piece;
  auto move = [&](U* __restrict__ c) {
    U v[W];
    bool on[W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
      on[j] = false;
      if (j < group) {
        const int from = source(src, lo + j, lo, group);
        on[j] = from != lo + j && pos >= (first ? first[lo + j] : 0) && pos < min(seq_lens[from], max_seq);
        v[j] = U{};
        if (on[j]) v[j] = c[at + from * seq];
      }
    }
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (j < group && on[j]) c[at + (lo + j) * seq] = v[j];
  };
  move(kc);
  move(vc);
}

// In a launch of its own: the one before reads the lengths in every workgroup.
__global__ void __launch_bounds__(64) k_reorder_lens(const int32_t* __restrict__ src, int group, int32_t* seq_lens) {
  const int lo = blockIdx.x * group, lane = threadIdx.x;
  int n = 0;
  if (lane < group) n = seq_lens[source(src, lo + lane, lo, group)];
  if (lane < group) seq_lens[lo + lane] = n;
}

template <class U>
void launch_reorder(const int32_t* src, const int32_t* first, int32_t* seq_lens, int groups, int group, int layers, int max_batch, int hkv, int max_seq,
                    int max_ctx, int pieces, void* kc, void* vc, hipStream_t st) {
  const dim3 grid((unsigned)(((size_t)max_ctx * pieces + 255) / 256), layers * hkv, groups);
#define LS_REORDER(w)                                                                                                                    \
  if (group <= w) {                                                                                                                      \
    k_reorder<w, U><<<grid, 256, 0, st>>>(src, first, seq_lens, group, max_batch, hkv, max_seq, pieces, (U*)kc, (U*)vc);                 \
    return;                                                                                                                              \
  }
  LS_REORDER(4) LS_REORDER(8) LS_REORDER(16) LS_REORDER(32) LS_REORDER(64)
#undef LS_REORDER
}

}  // namespace

}  // namespace ls

namespace {

using ls::bad;
using ls::launched;

bool select_ok(int groups, int beams, int vocab, int k) {
  return groups >= 1 && groups <= (1 << 24) && beams >= 1 && beams <= LS_BEAMS_MAX && vocab >= 1 && vocab <= (1 << 24) && k >= 1 &&
         k <= LS_BEAMS_MAX && (long)k <= (long)beams * vocab && (long)groups * beams <= INT32_MAX;
}

}  // namespace

extern "C" {

size_t ls_beam_select_scratch_bytes(int groups, int beams, int vocab, int k) { return select_ok(groups, beams, vocab, k) ? 256 : 0; }

ls_status ls_beam_select(const float* logits, const float* scores, const int32_t* ended, int groups, int beams, int vocab, int k, int eos,
                         int32_t* rows, int32_t* tokens, float* scores_out, void* scratch, size_t scratch_bytes, void* hip_stream) {
  static const char* who = "ls_beam_select";
  if (!logits || !scores || !rows || !tokens || !scores_out || !scratch) return bad(who, "NULL argument");
  if (!select_ok(groups, beams, vocab, k)) return bad(who, "beams and k are 1 to 64, k at most beams * vocab, groups and vocab at most 2^24");
  if (ended && (eos < 0 || eos >= vocab)) return bad(who, "eos outside the vocabulary");
  if (((uintptr_t)logits | (uintptr_t)scores) & 3) return bad(who, "a buffer is not aligned to its type");
  if ((uintptr_t)scratch & 15) return bad(who, "scratch is not aligned to 16 bytes");
  if (scratch_bytes < ls_beam_select_scratch_bytes(groups, beams, vocab, k)) {
    ls::set_last_error("%s: scratch too small", who);
    return LS_ERR_OOM;
  }
  ls::k_beam_select<<<groups, 1024, 0, (hipStream_t)hip_stream>>>(logits, scores, ended, beams, vocab, k, eos, rows, tokens, scores_out);
  return launched(who);
}

ls_status ls_kv_reorder(const ls_heads* h, int layers, const int32_t* src, int batch, int group, const int32_t* first, int max_ctx, const ls_kv* kv,
                        void* hip_stream) {
  static const char* who = "ls_kv_reorder";
  if (const char* e = ls::heads_error(h)) return bad(who, e);
  if (!src || !kv || !kv->k || !kv->v || !kv->seq_lens) return bad(who, "NULL argument");
  if (batch < 1 || batch > (int)h->max_batch) return bad(who, "batch outside [1, max_batch]");
  if (group < 1 || group > LS_BEAMS_MAX || batch % group || batch / group > 65535) return bad(who, "group has to be 1 to 64 and divide batch into at most 65535");
  if (max_ctx < 0 || max_ctx > (int)h->max_seq) return bad(who, "max_ctx outside [0, max_seq]");
  if (layers < 1 || (long)layers * h->n_kv_heads > 65535) return bad(who, "layers * n_kv_heads outside [1, 65535]");
  if (((uintptr_t)kv->k | (uintptr_t)kv->v) & 3) return bad(who, "a cache is not aligned to 4 bytes");
  hipStream_t st = (hipStream_t)hip_stream;
  const size_t row = (size_t)h->head_dim * (h->dtype == LS_DTYPE_F32 ? 4 : 2);
  const bool wide = row % 16 == 0 && (((uintptr_t)kv->k | (uintptr_t)kv->v) & 15) == 0;
  if (group == 1) return LS_OK;
  if (max_ctx > 0) {
    if (wide)
      ls::launch_reorder<ls::u32x4>(src, first, kv->seq_lens, batch / group, group, layers, (int)h->max_batch, (int)h->n_kv_heads, (int)h->max_seq, max_ctx,
                                (int)(row / 16), kv->k, kv->v, st);
    else
      ls::launch_reorder<uint32_t>(src, first, kv->seq_lens, batch / group, group, layers, (int)h->max_batch, (int)h->n_kv_heads, (int)h->max_seq,
                                   max_ctx, (int)(row / 4), kv->k, kv->v, st);
  }
  ls::k_reorder_lens<<<batch / group, 64, 0, st>>>(src, group, kv->seq_lens);
  return launched(who);
}

}  // extern "C"
