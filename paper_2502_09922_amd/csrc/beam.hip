// Beam search beside a stage: the k best continuations of each request's beams, and the caches' reordering behind them.
#include "entry.hpp"
#include "device_util.hpp"

#include <algorithm>

namespace ls {

namespace {

constexpr int BEAMS_MAX = LS_BEAMS_MAX;

// ---- selection in two launches.
//
// k_beam_rows reads the logits once.  A row is cut into segments of SEG tokens, a workgroup to each; a thread's EACH tokens of a segment
// (float4s 256 apart), or four neighbours' together, are a set of which it leaves the largest logit and its float4, the segment leaves
// its maximum and its sum of exponentials.  k_beam_pick, a workgroup to a request, makes scores of them: the k best candidates of a request lie in the k
// sets whose best ones are the best, for a candidate of another set has k better ones in front of it.  It chooses those sets and reads
// their logits again, k x EACH (x 4) of beams x vocab.
//
// Order: the higher score; of equal ones the lower beam, the larger logit, the lower token.  Within a beam that is the order of the
// logits, so that a set's best is known before its row's sum is.
//
// Bound by the one reading: 64 x 5 rows of 50257 tokens (64 MB) 13.4 us, 4.8 TB/s; the choice 8.4, most of it waits one after the
// other (sums, bound, sets, tokens), 6.0 for one request.
constexpr int SEG = 8192, EACH = SEG / 256;
constexpr int HELD = 12288;            // sets in LDS: what 5 beams of 64k tokens leave, four times as many for up to 16 candidates
constexpr int LIST = 2048;             // candidates in LDS: >= BEAMS_MAX * EACH, 16 * 4 EACH
constexpr float LOG2E = 1.4426950408889634f;

// Sets of a segment, as a power of two: those of four threads together for up to 16 candidates, whose sets' tokens then still fit LIST.
// 8 requests of 8 beams of 128256 tokens, 16 candidates 18.0 us, 31.7 with a set to a thread; 64 of 5 of 50257, 10 candidates 20.4 and 22.5.
__host__ __device__ constexpr int set_bits(int k) { return k <= 16 ? 6 : 8; }

struct Set {
  float m;  // the largest logit of its tokens
  int at;   // the first token of the float4 that has it
};
struct SegSum {
  double l;  // sum of exp(x - m)
  float m;
  int pad;
};
struct Cand {
  double s;  // score
  float x;   // logit
  int at;    // beam << 24 | token
};
constexpr int NONE = 0x7fffffff;  // Cand::at of no candidate
__device__ __forceinline__ bool before(Cand a, Cand b) {
  if (a.s != b.s) return a.s > b.s;
  if (a.at >> 24 != b.at >> 24 || a.x == b.x) return a.at < b.at;
  return a.x > b.x;
}
__device__ __forceinline__ Cand cand_xor(Cand c, int off) {
  Cand o;
  o.s = __shfl_xor(c.s, off);
  o.x = __shfl_xor(c.x, off);
  o.at = __shfl_xor(c.at, off);
  return o;
}

__global__ void __launch_bounds__(256)
k_beam_rows(const float* __restrict__ logits, const int32_t* __restrict__ ended, int vocab, int nseg, int bits, Set* __restrict__ sets, SegSum* __restrict__ sums) {
  typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));  // a row may start anywhere
  const int row = blockIdx.x, seg = blockIdx.y, tid = threadIdx.x;
  if (ended && ended[row]) return;  // its logits are not used
  const float* x = logits + (size_t)row * vocab;
  const int first = seg * SEG + tid * 4;
  f32x4 v[EACH / 4];
#pragma unroll
  for (int j = 0; j < EACH / 4; ++j) {
    const int at = first + j * 1024;
    v[j] = f32x4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if (at + 4 <= vocab) {
      v[j] = *reinterpret_cast<const f32x4u*>(x + at);
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (at + e < vocab) v[j][e] = x[at + e];
    }
  }
  float m = -INFINITY;
  int best = first;
#pragma unroll
  for (int j = 0; j < EACH / 4; ++j) {
    const float mj = fmaxf(fmaxf(v[j][0], v[j][1]), fmaxf(v[j][2], v[j][3]));
    if (mj > m) {
      m = mj;
      best = first + j * 1024;
    }
  }
  if (bits == 8) {
    sets[((size_t)row * nseg + seg) * 256 + tid] = Set{m, best};
  } else {  // of equal ones the lowest
    float m4 = m;
    int best4 = best;
#pragma unroll
    for (int off = 1; off < 4; off *= 2) {
      const float mo = __shfl_xor(m4, off);
      const int bo = __shfl_xor(best4, off);
      if (mo > m4 || (mo == m4 && bo < best4)) {
        m4 = mo;
        best4 = bo;
      }
    }
    if ((tid & 3) == 0) sets[((size_t)row * nseg + seg) * 64 + (tid >> 2)] = Set{m4, best4};
  }
  // sums behind the workgroup's maximum; the difference before the product, whose rounding then is each addend's own
  __shared__ float top[4];
  __shared__ double part[4];
  float M = exchange<32, 1>(m, Max{});
  if ((tid & 63) == 0) top[tid >> 6] = M;
  __syncthreads();
  M = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
  const float ref = M == -INFINITY ? 0.f : M;
  float l = 0.f;
#pragma unroll
  for (int j = 0; j < EACH / 4; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) l += __builtin_amdgcn_exp2f((v[j][e] - ref) * LOG2E);
  double s = l;
#pragma unroll
  for (int off = 32; off; off >>= 1) s += __shfl_xor(s, off);
  if ((tid & 63) == 0) part[tid >> 6] = s;
  __syncthreads();
  if (tid == 0) sums[(size_t)row * nseg + seg] = SegSum{(part[0] + part[1]) + (part[2] + part[3]), M, 0};
}

__global__ void __launch_bounds__(1024)
k_beam_pick(const float* __restrict__ logits, const float* __restrict__ scores, const int32_t* __restrict__ ended, int beams, int vocab, int k, int eos,
            int nseg, unsigned nseg_inv, int bits, const Set* __restrict__ sets, const SegSum* __restrict__ sums, int32_t* __restrict__ rows_out, int32_t* __restrict__ tokens,
            float* __restrict__ scores_out) {
  constexpr int NT = 1024;
  enum { DEAD = 0, LIVE = 1, ENDED = 2 };
  __shared__ double base[BEAMS_MAX];  // score - log(sum)
  __shared__ float most[BEAMS_MAX];   // the largest logit; of an ended beam the score
  __shared__ int state[BEAMS_MAX], chosen[BEAMS_MAX], count;
  __shared__ Cand some[64], bound, list[LIST];
  __shared__ int id[LIST];
  __shared__ int rank[LIST];
  struct Rough {  // a beam in 32 bits
    float most, base, score;
    int eos_set;  // of an ended beam
  };
  __shared__ Rough rough[BEAMS_MAX];
  __shared__ __attribute__((aligned(16))) float part[64];
  __shared__ float rough_bound;
  const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const size_t row0 = (size_t)g * beams;
  const int C = nseg << bits, N = beams * C;
  const int wide = 10 - bits, each_set = 13 - bits;  // neighbouring tokens of a set, all of its tokens, as powers of two
  static_assert(SEG == 1 << 13, "");
  auto beam_of = [&](int e) { return (int)__umulhi((unsigned)(e >> bits) * 2u, nseg_inv); };
  auto first_of = [&](int c) { return (c >> bits) * SEG + ((c & ((1 << bits) - 1)) << wide); };  // of the c-th set of a row
  const int eos_at = (eos / SEG << bits) + ((eos & 1023) >> wide);  // the set that holds it
  const Set* mine_sets = sets + row0 * C;
  // Sets go through LDS, HELD at a time: all on their way at once, and then short loops.  (The loops unrolled: 18.4 us for 64 x 5 beams
  // instead of 15.1.)
  __shared__ Set held[HELD];
  auto load = [&](int e0) {
    Set v[HELD / NT];
#pragma unroll
    for (int u = 0; u < HELD / NT; ++u)
      if (e0 + u * NT < N) v[u] = mine_sets[min(e0 + u * NT + tid, N - 1)];
#pragma unroll
    for (int u = 0; u < HELD / NT; ++u)
      if (e0 + u * NT < N) held[u * NT + tid] = v[u];
  };
  load(0);
  {  // sixteen threads to a beam
    const int beam = tid >> 4;
    const bool in = beam < beams;
    const size_t r = row0 + (in ? beam : 0);
    const bool end = ended && ended[r];
    const float score = scores[r];
    float M = -INFINITY;
    for (int s = tid & 15; s < nseg; s += 16) M = fmaxf(M, sums[r * nseg + s].m);
    M = exchange<8, 1>(M, Max{});
    double l = 0.;
    for (int s = tid & 15; s < nseg; s += 16) {
      const SegSum p = sums[r * nseg + s];
      l += p.m == -INFINITY ? p.l : p.l * exp((double)p.m - (double)M);
    }
#pragma unroll
    for (int off = 8; off; off >>= 1) l += __shfl_xor(l, off);
    if (in && (tid & 15) == 0) {
      const double b = (double)score - log(l);
      // dead: nothing left of the logits, or one that makes the sum none; such have no candidate above -inf
      if (end) state[beam] = score < INFINITY && score > -INFINITY ? ENDED : DEAD;
      else state[beam] = M < INFINITY && M > -INFINITY && b < INFINITY && b > -INFINITY ? LIVE : DEAD;
      base[beam] = b;
      most[beam] = end ? score : M;
      const bool live = state[beam] == LIVE, over = state[beam] == ENDED;
      rough[beam] = Rough{live ? M : 0.f, live ? (float)b : -INFINITY, score, over ? beam * C + eos_at : -1};
    }
  }
  if (tid == 0) {
    count = 0;
    rough_bound = -INFINITY;
  }
  if (tid < 64) rank[tid] = 0;
  __syncthreads();

  auto score_of = [&](int beam, float x, int token) {
    Cand c{-INFINITY, 0.f, beam << 24 | token};
    if (state[beam] == LIVE) {
      c.s = ((double)x - (double)most[beam]) + base[beam];  // x apart from the rest: next to a large one that would be lost
      c.x = x;
    } else if (state[beam] == ENDED && token == eos) {
      c.s = most[beam];
    }
    return c;
  };
  // the best of set e.  Its token is that of a float4: sets share none, so that it orders them
  auto best_of = [&](int e, Set s) {
    const int beam = beam_of(e), c = e - beam * C, first = first_of(c);
    if (first >= vocab) return Cand{-INFINITY, 0.f, NONE};
    if (state[beam] == LIVE) return score_of(beam, s.m, s.at);
    return score_of(beam, 0.f, state[beam] == ENDED && c == eos_at ? eos : first);
  };
  // f(set, what it left) for all of this thread's: it reads what it has written itself
  auto each = [&](auto f) {
    for (int e0 = 0; e0 < N; e0 += HELD) {
      if (N > HELD) load(e0);
#pragma unroll 1
      for (int e = tid; e < min(HELD, N - e0); e += NT) f(e0 + e, held[e]);
    }
  };
  // rank[i] += how many of n candidates stand before the one at i, a copy in front of it included; a sixteenth of them to a wavefront
  auto add_ranks = [&](const Cand* of, int n) {
    for (int i = lane; i < n; i += 64) {
      const Cand c = of[i];
      int r = 0;
      for (int j = tid >> 6; j < n; j += NT / 64) {
        const Cand o = of[j];
        r += o.s > c.s;
        if (o.s == c.s && i != j) r += before(o, c) || (j < i && !before(c, o));
      }
      if (r) atomicAdd(&rank[i], r);
    }
  };

  auto push = [&](int e, Cand c) {
    const int to = atomicAdd(&count, 1);
    if (to < LIST) {
      list[to] = c;
      id[to] = e;
      rank[to] = 0;
    }
  };
  // ---- a bound: the k-th best of 64 parts' best sets; then the sets that are no worse.  In 32 bits with room for their rounding, 2^-24
  // of the logit, the base (twice) and the sum each
  auto rounded = [&](int e, float m, float way) {  // 64 neighbouring sets are one beam's
    const Rough b = rough[beam_of(__builtin_amdgcn_readfirstlane(e))];
    const float f = (m - b.most) + b.base;
    return e == b.eos_set ? b.score : f + way * 0x1p-21f * (fabsf(f) + fabsf(b.base));  // of a dead beam NaN
  };
  // g(i, e) for this thread's sets, the i-th of those held, e of all
  auto rough_each = [&](int e0, auto g) {
    const int n = min(HELD, N - e0);
#pragma unroll 1
    for (int i = tid; i < n; i += NT) g(i, e0 + i);
  };
  float top = -INFINITY;
  for (int e0 = 0; e0 < N; e0 += HELD) {
    if (N > HELD) load(e0);
    rough_each(e0, [&](int i, int e) { top = fmaxf(top, rounded(e, held[i].m, -1.f)); });
  }
  top = exchange<8, 1>(top, Max{});
  if ((tid & 15) == 0) part[tid >> 4] = top;
  __syncthreads();
  {  // each wavefront compares all with four of them
    const float c = part[lane];
    const f32x4 o = reinterpret_cast<const f32x4*>(part)[tid >> 6];
    int r = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) r += o[j] > c || (o[j] == c && (tid >> 6) * 4 + j < lane);
    if (r) atomicAdd(&rank[lane], r);
  }
  __syncthreads();
  if (tid < 64) {
    if (rank[tid] == k - 1) rough_bound = part[tid];
    rank[tid] = 0;
  }
  __syncthreads();
  const float least_top = rough_bound;
  // Not by the rough bound: fewer parts than k with any candidate above -inf (the order of those at -inf counts), or more sets than LIST within
  // its rounding, as where most logits are one finite value that masks (8 requests of 8 beams of 128256 tokens but five at -1e9, 32 candidates:
  // 77 us so, 627 one after the other, 32 without masks)
  bool exactly = !(least_top > -INFINITY);
  if (!exactly) {
    for (int e0 = 0; e0 < N; e0 += HELD) {
      if (N > HELD) load(e0);
      unsigned good = 0;  // of this thread's HELD / NT
      rough_each(e0, [&](int i, int e) { good |= (unsigned)(rounded(e, held[i].m, 1.f) >= least_top) << (i / NT); });
      for (; good; good &= good - 1) {
        const int i = __builtin_ctz(good) * NT + tid;
        push(e0 + i, best_of(e0 + i, held[i]));
      }
    }
    __syncthreads();
    exactly = count > LIST;
    __syncthreads();
    if (exactly && tid == 0) count = 0;
  }
  if (exactly) {
    Cand mine{-INFINITY, 0.f, NONE};
    each([&](int e, Set s) {
      const Cand c = best_of(e, s);
      if (before(c, mine)) mine = c;
    });
#pragma unroll
    for (int off = 8; off; off >>= 1) {
      const Cand c = cand_xor(mine, off);
      if (before(c, mine)) mine = c;
    }
    if ((tid & 15) == 0) some[tid >> 4] = mine;
    __syncthreads();
    add_ranks(some, 64);
    __syncthreads();
    if (tid < 64 && rank[tid] == k - 1) bound = some[tid];
    __syncthreads();
    const Cand lowest = bound;
    each([&](int e, Set s) {
      const Cand c = best_of(e, s);
      if (c.at != NONE && !before(lowest, c)) push(e, c);
    });
  }
  __syncthreads();
  const int found = count, sel = min(found, k);
  if (found <= LIST) {
    add_ranks(list, found);
    __syncthreads();
    for (int i = tid; i < found; i += NT) {
      const int r = rank[i];
      if (r < sel) chosen[r] = id[i];
      if (r == sel - 1) bound = list[i];
    }
  } else {  // more than there is room for, as in many equal ones: one after the other
    __shared__ int at[16];
    Cand last{INFINITY, 0.f, -1};
    for (int j = 0; j < sel; ++j) {
      Cand mine{-INFINITY, 0.f, NONE};
      int set = -1;
      each([&](int e, Set s) {
        const Cand c = best_of(e, s);
        if (before(last, c) && before(c, mine)) {
          mine = c;
          set = e;
        }
      });
      for (int off = 32; off; off >>= 1) {
        const Cand c = cand_xor(mine, off);
        const int o = __shfl_xor(set, off);
        if (before(c, mine)) {
          mine = c;
          set = o;
        }
      }
      if (lane == 0) {
        some[tid >> 6] = mine;
        at[tid >> 6] = set;
      }
      __syncthreads();
      for (int w = 0; w < NT / 64; ++w)
        if (!before(mine, some[w])) {
          mine = some[w];
          set = at[w];
        }
      last = mine;
      if (tid == 0) {
        chosen[j] = set;
        bound = mine;
      }
      __syncthreads();
    }
  }
  __syncthreads();
  if (tid == 0) count = 0;
  __syncthreads();

  // ---- the tokens of the chosen sets: the k-th best set's best one bounds the k-th best token
  Cand least = bound;
  least.at |= 3;  // the last token of its float4 that may be it
  for (int i = tid; i < sel << each_set; i += NT) {
    const int e = chosen[i >> each_set], q = i & ((1 << each_set) - 1);
    const int beam = beam_of(e), token = first_of(e - beam * C) + (q >> wide) * 1024 + (q & ((1 << wide) - 1));
    if (token >= vocab) continue;
    const Cand d = score_of(beam, state[beam] == LIVE ? logits[(row0 + beam) * vocab + token] : 0.f, token);
    if (sel < k || !before(least, d)) {
      const int to = atomicAdd(&count, 1);
      list[to] = d;
      rank[to] = 0;
    }
  }
  __syncthreads();
  const int n = count;
  add_ranks(list, n);
  __syncthreads();
  for (int i = tid; i < n; i += NT) {
    const int r = rank[i];
    if (r < k) {
      const size_t to = (size_t)g * k + r;
      rows_out[to] = (int)row0 + (list[i].at >> 24);
      tokens[to] = list[i].at & 0xffffff;
      scores_out[to] = (float)list[i].s;
    }
  }
}

// Sequence src[b], if it is of b's group, else b itself.
__device__ __forceinline__ int source(const int32_t* __restrict__ src, int b, int lo, int group) {
  const int s = src[b];
  return s >= lo && s < lo + group ? s : b;
}

// The positions of a request's W sequences, W or fewer, in place: a thread has a U-sized piece of all of them in registers before
// it writes any.  Workgroups of a (layer, kv head) walk the positions that anybody moves, which the device alone knows, however many
// workgroups the host's bound of the lengths has made.
// Bound by memory: 13B, 8 x 4 beams of up to 1087 positions, four layers, 4.1 GB read and written at 5.6 TB/s, where a copy of 1 GiB
// moves 5.2.  Rows of 126 dims, in pieces of four bytes, 32 of 1087 positions all moved 1263 us, of 128 1109.
template <int W, class U>
__global__ void __launch_bounds__(256, 1)
k_reorder(const int32_t* __restrict__ src, const int32_t* __restrict__ first, const int32_t* __restrict__ seq_lens, int group, int max_batch, int hkv,
          int max_seq, int pieces, U* __restrict__ kc, U* __restrict__ vc) {
  const int lo = blockIdx.z * group, layer = blockIdx.y / hkv, kh = blockIdx.y % hkv;
  const size_t seq = (size_t)hkv * max_seq * pieces;
  const size_t head = ((size_t)layer * max_batch * hkv + kh) * max_seq * pieces;
  int from[W], p0[W], p1[W], start = max_seq, end = 0;
#pragma unroll
  for (int j = 0; j < W; ++j) {
    from[j] = lo + j;
    p0[j] = p1[j] = 0;
    if (j < group) {
      from[j] = source(src, lo + j, lo, group);
      if (from[j] != lo + j) {
        p0[j] = first ? max(first[lo + j], 0) : 0;
        p1[j] = min(seq_lens[from[j]], max_seq);
        if (p0[j] < p1[j]) {
          start = min(start, p0[j]);
          end = max(end, p1[j]);
        }
      }
    }
  }
  if (start >= end) return;
  const size_t u1 = (size_t)end * pieces;
  for (size_t u = (size_t)start * pieces + blockIdx.x * 256u + threadIdx.x; u < u1; u += (size_t)gridDim.x * 256) {
    const int pos = (int)((unsigned)u / (unsigned)pieces);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      U* const c = (half ? vc : kc) + head + u;
      U v[W];
#pragma unroll
      for (int j = 0; j < W; ++j) {
        v[j] = U{};
        if (pos >= p0[j] && pos < p1[j]) v[j] = c[from[j] * seq];
      }
#pragma unroll
      for (int j = 0; j < W; ++j)
        if (pos >= p0[j] && pos < p1[j]) c[(lo + j) * seq] = v[j];
    }
  }
}

// In a launch of its own: the one before reads the lengths in every workgroup.
__global__ void __launch_bounds__(64) k_reorder_lens(const int32_t* __restrict__ src, int group, int32_t* seq_lens) {
  const int lo = blockIdx.x * group, lane = threadIdx.x;
  int n = 0;
  if (lane < group) n = seq_lens[source(src, lo + lane, lo, group)];
  if (lane < group) seq_lens[lo + lane] = n;
}

constexpr size_t MANY = 16384;

template <class U>
void launch_reorder(const int32_t* src, const int32_t* first, int32_t* seq_lens, int groups, int group, int layers, int max_batch, int hkv, int max_seq,
                    int max_ctx, int pieces, void* kc, void* vc, hipStream_t st) {
  // A workgroup for each 256 pieces below max_ctx where those are many, a quarter of that where it is few that have work (7B, four beams, 88
  // of 600 positions: 14.0 us, 18.1 with all; 13B, 8 x 4 beams: 760 and 735).  An odd number: ids go round the eight XCDs, and a number
  // of fours or eights leaves the few with work on some of them (10 of 100 positions, 256 heads: 12.8 us with 7, 22.5 with 8).
  const size_t blocks = ((size_t)std::max(max_ctx, 1) * pieces + 255) / 256, heads = (size_t)layers * hkv * groups;
  const dim3 grid((unsigned)(std::min<size_t>(blocks * heads > MANY ? blocks : (blocks + 3) / 4, 1 << 20) | 1), layers * hkv, groups);
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
  return groups >= 1 && groups < (1 << 22) && beams >= 1 && beams <= LS_BEAMS_MAX && vocab >= 1 && vocab <= (1 << 24) && k >= 1 &&
         k <= LS_BEAMS_MAX && (long)k <= (long)beams * vocab && (long)groups * beams < (1 << 24);
}

}  // namespace

extern "C" {

size_t ls_beam_select_scratch_bytes(int groups, int beams, int vocab, int k) {
  if (!select_ok(groups, beams, vocab, k)) return 0;
  return (size_t)groups * beams * ((vocab + ls::SEG - 1) / ls::SEG) * ((sizeof(ls::Set) << ls::set_bits(k)) + sizeof(ls::SegSum));
}

ls_status ls_beam_select(const float* logits, const float* scores, const int32_t* ended, int groups, int beams, int vocab, int k, int eos,
                         int32_t* rows, int32_t* tokens, float* scores_out, void* scratch, size_t scratch_bytes, void* hip_stream) {
  static const char* who = "ls_beam_select";
  if (!logits || !scores || !rows || !tokens || !scores_out || !scratch) return bad(who, "NULL argument");
  if (!select_ok(groups, beams, vocab, k)) return bad(who, "beams and k are 1 to 64, k at most beams * vocab, groups below 2^22, rows below 2^24, vocab 2^24 at most");
  if (ended && (eos < 0 || eos >= vocab)) return bad(who, "eos outside the vocabulary");
  if (((uintptr_t)logits | (uintptr_t)scores) & 3) return bad(who, "a buffer is not aligned to its type");
  if ((uintptr_t)scratch & 15) return bad(who, "scratch is not aligned to 16 bytes");
  if (scratch_bytes < ls_beam_select_scratch_bytes(groups, beams, vocab, k)) {
    ls::set_last_error("%s: scratch too small", who);
    return LS_ERR_OOM;
  }
  const int nseg = (vocab + ls::SEG - 1) / ls::SEG, n = groups * beams;
  ls::SegSum* sums = (ls::SegSum*)scratch;
  ls::Set* sets = (ls::Set*)(sums + (size_t)n * nseg);
  // x / nseg = umulhi(2 x, nseg_inv) for the x < 64 nseg there are, nseg <= 2048: the product is off by less than x nseg < 2^31
  const unsigned nseg_inv = (unsigned)(((1ull << 31) + nseg - 1) / nseg);
  const int bits = ls::set_bits(k);
  hipStream_t st = (hipStream_t)hip_stream;
  ls::k_beam_rows<<<dim3(n, nseg), 256, 0, st>>>(logits, ended, vocab, nseg, bits, sets, sums);
  ls::k_beam_pick<<<groups, 1024, 0, st>>>(logits, scores, ended, beams, vocab, k, eos, nseg, nseg_inv, bits, sets, sums, rows, tokens, scores_out);
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
  if (wide)
    ls::launch_reorder<ls::u32x4>(src, first, kv->seq_lens, batch / group, group, layers, (int)h->max_batch, (int)h->n_kv_heads, (int)h->max_seq, max_ctx,
                                  (int)(row / 16), kv->k, kv->v, st);
  else
    ls::launch_reorder<uint32_t>(src, first, kv->seq_lens, batch / group, group, layers, (int)h->max_batch, (int)h->n_kv_heads, (int)h->max_seq,
                                 max_ctx, (int)(row / 4), kv->k, kv->v, st);
  ls::k_reorder_lens<<<batch / group, 64, 0, st>>>(src, group, kv->seq_lens);
  return launched(who);
}

}  // extern "C"
