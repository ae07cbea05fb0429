// bf16 attention of draft trees on the matrix cores (head_dim 64 and 128).
//
// Nodes x query heads of a kv head are the columns of both products, all of which see the cached keys:
//   S^T[key][column] = K Q^T        v_mfma_f32_16x16x32_bf16, A = 16 key rows, B = 16 columns
//   O^T[dim][column] += V^T P^T     A = V^T by transposing LDS reads of the row-major tile, B = P^T
// A lane of a result holds column lane % 16 and rows 4 (lane / 16) + e: one column's running maximum and sum are per-lane values
// and exchanges with lanes +-16 and +-32, and the eight weights a lane has for 32 keys are a B operand whose k index runs over
// keys {4g..4g+3, 16+4g..16+4g+3}, g = lane / 16.
//
// Queries are turned in fp32 and enter as a sum of two bf16 (16 bits and more of them): rounded once they would move every score by
// 2^-9 of its size, which costs more than the rounding of the output.  Weights are rounded to bf16 for the second product (their
// sum is of the unrounded ones), as the prompt kernel does.
//
// A workgroup is a (sequence, kv head, block of columns, chunk of keys).  Of its four wavefronts CW share keys, each with columns
// of its own, and 4 / CW split the chunk's keys.  Up to 16 columns each walks keys of its own, 32 at a time through registers into LDS of
// its own, no barriers (CW = 1); wavefronts that share keys fill double-buffered tiles together.  The splits' results are joined
// through LDS, chunks' by a second kernel, both in order.
//
// The nodes' own rows are turned, rounded and written to their slots by whoever reads those, a wavefront (CW = 1) or a workgroup,
// before it reads them: blocks of columns write the same bytes, and none depends on another workgroup's.  Only in the tiles of
// those slots columns see different keys.
#include "tree.hpp"

#include <algorithm>

namespace ls {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// 16-byte chunks of a row of a tile are permuted by its key, so that 16 rows' equal chunks (keys) and 4 rows' 32 bytes (values,
// transposing) lie in different banks.
template <int HD> __device__ __forceinline__ int key_swizzle(int key) { return HD == 128 ? key & 15 : ((key & 3) << 1) | ((key >> 2) & 1); }
template <int HD> __device__ __forceinline__ int value_swizzle(int key) { return HD == 128 ? (key & 7) << 1 : ((key & 3) << 1) | ((key >> 2) & 1); }

// Values that are no numbers become zeros; whether there were any.
__device__ __forceinline__ bool drop_nonfinite(u32x4& v) {
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = (v[i] & 0x7F80u) == 0x7F80u, hi = (v[i] & 0x7F800000u) == 0x7F800000u;
    any |= lo || hi;
    v[i] &= (lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u);
  }
  return any;
}

constexpr int SM_PAD = 4;  // floats behind a column's output in LDS: 16 columns' equal dims in different banks

// Steps of 32 keys in a tile: two where tiles are shared by all and the registers suffice.
template <int HD, int CT, int CW> constexpr int steps_of() { return CW == 4 && (CT == 1 || HD == 64) ? 2 : 1; }

template <int HD, int CT, int CW>
__global__ void __launch_bounds__(256, 2)
k_tree_mfma(const int32_t* __restrict__ cu, const int32_t* __restrict__ seq_lens, const int32_t* __restrict__ parents, const bf16* __restrict__ qkv,
            const float* __restrict__ cs, bf16* __restrict__ kc, bf16* __restrict__ vc, bf16* __restrict__ out, int rows, int hq, int hkv, int max_seq,
            int nchunk, int chunk_tiles, float* __restrict__ part_o, float2* __restrict__ part_ml) {
  constexpr int KW = 4 / CW;             // wavefronts that split the keys
  constexpr int SUB = steps_of<HD, CT, CW>();
  constexpr int TK = 32 * SUB;
  constexpr int ROWB = HD * 2;
  constexpr int CPR = HD / 8;            // 16-byte chunks of a row
  constexpr int RPI = 64 / CPR;          // rows that a wavefront's load covers
  constexpr int NL = TK / RPI / CW;      // loads of a wavefront for a tile's keys, as many for its values
  constexpr int TILE = TK * ROWB;
  constexpr int COLS = 16 * CT * CW;     // of a workgroup
  constexpr int KS = HD / 32, DT = HD / 16;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];

  const int G = hq / hkv;
  const int b = blockIdx.z, kh = blockIdx.y % hkv, cb = blockIdx.y / hkv, z = blockIdx.x;
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  TreeSeq t;
  const bool room = tree_seq(cu, seq_lens, b, rows, max_seq, t);
  if (t.n <= 0 || t.n > TREE_MAX || t.row0 < 0 || t.row0 > rows - t.n || cb * COLS >= t.n * G) return;
  if (!room) {  // the rows hold zeros
    if (z == 0 && cb == 0)
      for (int i = threadIdx.x; i < t.n * G * HD; i += 256) {
        const int c = i / HD;
        out[((size_t)(t.row0 + c / G) * hq + kh * G + c % G) * HD + i % HD] = (bf16)0.f;
      }
    return;
  }
  const int keys = t.ctx + t.n;
  const int ntile = (keys + TK - 1) / TK;
  const int t_lo = z * chunk_tiles;
  if (t_lo >= ntile) return;
  // the last chunk takes what is left, should the caller have understated the longest context
  const int t_hi = z == nchunk - 1 ? ntile : min(t_lo + chunk_tiles, ntile);
  const int per = (t_hi - t_lo + KW - 1) / KW;
  const int split = wave / CW, share = wave % CW;  // of the keys, of the columns and a tile's rows
  const int t_begin = min(t_lo + split * per, t_hi), t_end = min(t_begin + per, t_hi);

  const size_t head0 = ((size_t)b * hkv + kh) * max_seq * HD;
  bf16 *kb = kc + head0, *vb = vc + head0;
  const int stride = (hq + 2 * hkv) * HD;
  const bf16* rows0 = qkv + (size_t)t.row0 * stride;
  const int lrow = lane / CPR, lchunk = lane % CPR;
  const int first_row = share * NL * RPI;  // of a tile, that this wavefront brings

  u32x4 kreg[NL], vreg[NL];
  auto load = [&](int tile) {  // rows' byte offsets are of 32 bits behind the tile's address
    const int row0 = tile * TK + first_row;
    const char *kt = (const char*)(kb + (size_t)row0 * HD), *vt = (const char*)(vb + (size_t)row0 * HD);
    auto fetch = [&](int i, int from) {
      const int r = first_row + i * RPI + lrow;
      const u32x4* kp = reinterpret_cast<const u32x4*>(kt + from * ROWB + (unsigned)((lchunk ^ key_swizzle<HD>(r)) << 4));
      const u32x4* vp = reinterpret_cast<const u32x4*>(vt + from * ROWB + (unsigned)((lchunk ^ value_swizzle<HD>(r)) << 4));
      kreg[i] = CW == 1 ? __builtin_nontemporal_load(kp) : *kp;
      vreg[i] = CW == 1 ? __builtin_nontemporal_load(vp) : *vp;
    };
    if ((tile + 1) * TK <= keys) {
#pragma unroll
      for (int i = 0; i < NL; ++i) fetch(i, i * RPI + lrow);
    } else {  // rows behind the last key: that one again, which their weights of zero leave out
#pragma unroll
      for (int i = 0; i < NL; ++i) fetch(i, min(i * RPI + lrow, keys - 1 - row0));
    }
  };
  const bool early = t_begin < t_end && (t_begin + 1) * TK <= t.ctx;
  if (early) load(t_begin);  // on its way while nodes and queries are made ready

  const uint64_t path = tree_path(parents, t);
  {  // the nodes' rows among the keys of this wavefront (CW = 1) or workgroup
    const int depth = __builtin_popcountll(path) - 1;
    const int n_lo = max((CW == 1 ? t_begin : t_lo) * TK, t.ctx), items = (min((CW == 1 ? t_end : t_hi) * TK, keys) - n_lo) * CPR;
    constexpr int STEP = CW == 1 ? 64 : 256;
    for (int i0 = 0; i0 < items; i0 += STEP) {
      const int i = i0 + (CW == 1 ? lane : (int)threadIdx.x), key = n_lo + i / CPR, ch = i % CPR, node = min(key - t.ctx, t.n - 1);
      const int d = __shfl(depth, node);
      if (i < items) {
        const bf16* row = rows0 + (size_t)node * stride + ch * 8;
        u32x4 k = *reinterpret_cast<const u32x4*>(row + (size_t)(hq + kh) * HD);
        const u32x4 v = *reinterpret_cast<const u32x4*>(row + (size_t)(hq + hkv + kh) * HD);
        if (cs) {
          const bf16x8 u = __builtin_bit_cast(bf16x8, k);
          const f32x4* turn = reinterpret_cast<const f32x4*>(cs + (size_t)(t.ctx + d) * HD + ch * 8);
          const f32x4 ta = turn[0], tb = turn[1];
          bf16x8 w;
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const float2 c2 = p < 2 ? float2{ta[2 * p], ta[2 * p + 1]} : float2{tb[2 * p - 4], tb[2 * p - 3]};
            w[2 * p] = (bf16)turn0((float)u[2 * p], (float)u[2 * p + 1], c2);
            w[2 * p + 1] = (bf16)turn1((float)u[2 * p], (float)u[2 * p + 1], c2);
          }
          k = __builtin_bit_cast(u32x4, w);
        }
        *reinterpret_cast<u32x4*>(kb + (size_t)key * HD + ch * 8) = k;
        *reinterpret_cast<u32x4*>(vb + (size_t)key * HD + ch * 8) = v;
      }
    }
    if constexpr (CW == 1) {
      if (items > 0) __threadfence_block();  // other lanes of this wavefront read them
    } else {
      __syncthreads();
    }
  }

  // ---- this wavefront's columns: queries as two bf16 parts, the nodes they see
  const int col0 = cb * COLS + share * 16 * CT + lr;
  bf16x8 qh[CT][KS], ql[CT][KS];
  uint64_t sees[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    const int col = col0 + 16 * c;
    const bool in = col < t.n * G;
    const int node = in ? col / G : 0;
    sees[c] = (uint64_t)(unsigned)__shfl((int)(unsigned)(path >> 32), node) << 32 | (unsigned)__shfl((int)(unsigned)path, node);
    const int pos = t.ctx + __builtin_popcountll(sees[c]) - 1;
    const bf16* q = rows0 + (size_t)node * stride + (size_t)(kh * G + (in ? col % G : 0)) * HD;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      const int d0 = kk * 32 + lg * 8;
      const bf16x8 raw = *reinterpret_cast<const bf16x8*>(q + d0);
      float turn[8];
      if (cs) {
        const f32x4* cp = reinterpret_cast<const f32x4*>(cs + (size_t)pos * HD + d0);
        *reinterpret_cast<f32x4*>(turn) = cp[0];
        *reinterpret_cast<f32x4*>(turn + 4) = cp[1];
      }
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        float u0 = (float)raw[2 * p], u1 = (float)raw[2 * p + 1];
        if (cs) {
          const float2 c2{turn[2 * p], turn[2 * p + 1]};
          const float w0 = turn0(u0, u1, c2), w1 = turn1(u0, u1, c2);
          u0 = w0;
          u1 = w1;
        }
        qh[c][kk][2 * p] = (bf16)u0;
        qh[c][kk][2 * p + 1] = (bf16)u1;
        ql[c][kk][2 * p] = (bf16)(u0 - (float)qh[c][kk][2 * p]);
        ql[c][kk][2 * p + 1] = (bf16)(u1 - (float)qh[c][kk][2 * p + 1]);
      }
    }
  }

  f32x4 o[CT][DT];
  float m_run[CT], l_run[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) {
    m_run[c] = -INFINITY;
    l_run[c] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[c][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float scale = 1.4426950408889634f / sqrtf((float)HD);  // score -> exponent of 2

  // ---- 32 keys of a tile in LDS
  auto attend = [&](const unsigned char* ks, const unsigned char* vs, int sub, int key0, bool odd) {
    f32x4 s[CT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int kl = sub * 32 + h * 16 + lr;
#pragma unroll
      for (int c = 0; c < CT; ++c) s[c][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(ks + kl * ROWB + (((kk * 4 + lg) ^ key_swizzle<HD>(kl)) << 4));
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          s[c][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, ql[c][kk], s[c][h], 0, 0, 0);
          s[c][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qh[c][kk], s[c][h], 0, 0, 0);
        }
      }
    }
    bf16x8 pf[CT];
    const int behind = key0 - t.ctx;  // of the cached positions
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      if (behind > -32) {  // slots of nodes
        const unsigned seen = behind >= 64 ? 0u : behind >= 0 ? (unsigned)(sees[c] >> behind) : (unsigned)(sees[c] << -behind) | ((1u << -behind) - 1u);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[c][h][e] = seen >> (h * 16 + 4 * lg + e) & 1u ? s[c][h][e] : -INFINITY;
      }
      float mx = fmaxf(fmaxf(fmaxf(s[c][0][0], s[c][0][1]), fmaxf(s[c][0][2], s[c][0][3])), fmaxf(fmaxf(s[c][1][0], s[c][1][1]), fmaxf(s[c][1][2], s[c][1][3])));
      mx = exchange<16, 32>(mx, Max{});
      const float m_new = fmaxf(m_run[c], mx), m_ref = m_new == -INFINITY ? 0.f : m_new;
      if (__builtin_amdgcn_ballot_w64(m_new > m_run[c]) != 0) {
        const float corr = __builtin_amdgcn_exp2f((m_run[c] - m_ref) * scale);
        l_run[c] *= corr;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[c][d][e] *= corr;
        m_run[c] = m_new;
      }
      const float mc = m_ref * scale;
      float sum = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[c][h][e], scale, -mc));
          sum += p;
          pf[c][h * 4 + e] = (bf16)p;
        }
      l_run[c] += sum;
    }
    const int k0 = sub * 32 + 4 * lg + (lr >> 2), k1 = k0 + 16;
    const int within = (lr & 1) * 8;  // of the 16-byte chunk that holds dims 4 (lr % 4) of 16
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const int ch = d * 2 + ((lr & 3) >> 1);
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vs + k0 * ROWB + ((ch ^ value_swizzle<HD>(k0)) << 4) + within));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vs + k1 * ROWB + ((ch ^ value_swizzle<HD>(k1)) << 4) + within));
      const bf16x8 vt = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int c = 0; c < CT; ++c) o[c][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pf[c], o[c][d], 0, 0, 0);
    }
    if (odd) {  // nodes' values that are no numbers lie in the tile as zeros: only the columns that see the nodes take them
      for (int j = max(0, -behind); j < 32 && behind + j < t.n; ++j) {
        const bf16* v = rows0 + (size_t)(behind + j) * stride + (size_t)(hq + hkv + kh) * HD + 4 * lg;
        const int from = ((j >> 2) & 3) * 16 + lr;
#pragma unroll
        for (int c = 0; c < CT; ++c) {
          float p = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) p = (j >> 4) * 4 + (j & 3) == i ? (float)pf[c][i] : p;
          p = __shfl(p, from);
          if (!(sees[c] >> (behind + j) & 1)) continue;
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const bf16x4 x = *reinterpret_cast<const bf16x4*>(v + d * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (!(fabsf((float)x[e]) < INFINITY)) o[c][d][e] += p * (float)x[e];
            __builtin_amdgcn_sched_barrier(0);  // rare: no registers for it
          }
        }
      }
    }
  };
  // registers -> LDS, lane by lane.  True if a node's value is no number: zero times it would be none in columns that do not see
  // the node.  (Values of cached positions are seen by all.)
  auto put = [&](unsigned char* ks, unsigned char* vs, int tile) {
    bool odd = false;
    if ((tile + 1) * TK > t.ctx) {
#pragma unroll
      for (int i = 0; i < NL; ++i)
        if (tile * TK + first_row + i * RPI + lrow >= t.ctx) odd |= drop_nonfinite(vreg[i]);
    }
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int at = (first_row + i * RPI) * ROWB + lane * 16;
      *reinterpret_cast<u32x4*>(ks + at) = kreg[i];
      *reinterpret_cast<u32x4*>(vs + at) = vreg[i];
    }
    return __builtin_amdgcn_ballot_w64(odd) != 0;
  };
  const bool whole = ntile <= chunk_tiles || nchunk == 1;  // the sequence is this one chunk: its output rows go out
  const size_t pieces = (size_t)z * rows * hq;
  auto row_of = [&](int col) { return (size_t)(t.row0 + col / G) * hq + kh * G + col % G; };

  __shared__ int odd_flags[2][4];
  unsigned char* tiles = smem + split * ((CW == 1 ? 1 : 2) * 2 * TILE);  // one buffer of keys and values, or two
  for (int i = t_begin - 1; i < t_begin + per; ++i) {  // tile i is attended to while i + 1 is on its way; as many turns for all
    if constexpr (CW == 1) {
      bool odd = false;
      if (i >= t_begin && i < t_end) odd = put(tiles, tiles + TILE, i);
      if (i + 1 < t_end && (i >= t_begin || !early)) load(i + 1);
      if (i >= t_begin && i < t_end) attend(tiles, tiles + TILE, 0, i * TK, odd);
    } else {
      const int buf = (i - t_begin) & 1;
      const unsigned char *ks = tiles + buf * (2 * TILE), *vs = ks + TILE;
      if (i + 1 < t_end && (i >= t_begin || !early)) load(i + 1);
      if (i >= t_begin && i < t_end) {
        int odd = 0;
#pragma unroll
        for (int w = 0; w < CW; ++w) odd |= odd_flags[buf][split * CW + w];
#pragma unroll 1
        for (int sub = 0; sub < SUB; ++sub)
          if (i * TK + sub * 32 < keys) attend(ks, vs, sub, i * TK + sub * 32, odd != 0);
      }
      if (i + 1 < t_end) {
        unsigned char* to = tiles + (buf ^ 1) * (2 * TILE);
        const bool odd = put(to, to + TILE, i + 1);
        if (lane == 0) odd_flags[buf ^ 1][wave] = odd;
      }
      __syncthreads();
    }
  }

  if constexpr (KW > 1) {  // ---- the splits' results, in their order
    __shared__ float sm_m[KW][COLS], sm_l[KW][COLS];
    __syncthreads();  // nobody reads tiles any more
    float* sm_o = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const float l = exchange<16, 32>(l_run[c], Add{});
      const int at = (share * CT + c) * 16 + lr;
      if (lg == 0) {
        sm_m[split][at] = m_run[c];
        sm_l[split][at] = l;
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(sm_o + (split * COLS + at) * (HD + SM_PAD) + d * 16 + 4 * lg) = o[c][d];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < COLS * (HD / 4); i += 256) {
      const int c = i / (HD / 4), d = i % (HD / 4) * 4, col = cb * COLS + c;
      if (col >= t.n * G) break;
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < KW; ++w) m = fmaxf(m, sm_m[w][c]);
      f32x4 num{0.f, 0.f, 0.f, 0.f};
      float den = 0.f;
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const float mw = sm_m[w][c], wt = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mw - m) * scale);
        const f32x4 v = *reinterpret_cast<const f32x4*>(sm_o + (w * COLS + c) * (HD + SM_PAD) + d);
#pragma unroll
        for (int e = 0; e < 4; ++e) num[e] += v[e] * wt;
        den += sm_l[w][c] * wt;
      }
      const size_t row = row_of(col);
      if (whole) {
        bf16x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (bf16)(num[e] / den);
        *reinterpret_cast<bf16x4*>(out + row * HD + d) = v;
      } else {
        *reinterpret_cast<f32x4*>(part_o + (pieces + row) * HD + d) = num;
        if (d == 0) part_ml[pieces + row] = float2{m, den};
      }
    }
  } else {
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const int col = col0 + 16 * c;
      const float l = exchange<16, 32>(l_run[c], Add{});
      if (col >= t.n * G) continue;
      const size_t row = row_of(col);
      if (whole) {
        const float inv = 1.0f / l;
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          bf16x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (bf16)(o[c][d][e] * inv);
          *reinterpret_cast<bf16x4*>(out + row * HD + d * 16 + 4 * lg) = v;
        }
      } else {
#pragma unroll
        for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(part_o + (pieces + row) * HD + d * 16 + 4 * lg) = o[c][d];
        if (lg == 0) part_ml[pieces + row] = float2{m_run[c], l};
      }
    }
  }
}

// Rows of sequences of several chunks: the chunks' results in chunk order, four dims to a thread.
template <int HD>
__global__ void __launch_bounds__(256)
k_tree_merge(const int32_t* __restrict__ cu, const int32_t* __restrict__ seq_lens, int rows, int hq, int max_seq, int nchunk, int chunk_keys,
             const float* __restrict__ part_o, const float2* __restrict__ part_ml, bf16* __restrict__ out) {
  constexpr int TPR = HD / 4;
  const int node = blockIdx.x, b = blockIdx.y, h = blockIdx.z * (256 / TPR) + threadIdx.x / TPR, d = threadIdx.x % TPR * 4;
  TreeSeq t;
  if (!tree_seq(cu, seq_lens, b, rows, max_seq, t) || node >= t.n || h >= hq) return;
  const int n = min((t.ctx + t.n + chunk_keys - 1) / chunk_keys, nchunk);
  if (n == 1) return;  // the first pass wrote these rows
  const float scale = 1.4426950408889634f / sqrtf((float)HD);
  const size_t row = (size_t)(t.row0 + node) * hq + h, step = (size_t)rows * hq;
  float m = -INFINITY;
#pragma unroll 8
  for (int z = 0; z < n; ++z) m = fmaxf(m, part_ml[row + z * step].x);
  f32x4 num{0.f, 0.f, 0.f, 0.f};
  float den = 0.f;
#pragma unroll 8
  for (int z = 0; z < n; ++z) {
    const float2 ml = part_ml[row + z * step];
    const float wt = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((ml.x - m) * scale);
    const f32x4 v = *reinterpret_cast<const f32x4*>(part_o + (row + z * step) * HD + d);
#pragma unroll
    for (int e = 0; e < 4; ++e) num[e] += v[e] * wt;
    den += ml.y * wt;
  }
  bf16x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (bf16)(num[e] / den);
  *reinterpret_cast<bf16x4*>(out + row * HD + d) = v;
}

template <int HD, int CT, int CW>
void launch(const TreeAttn& a, const TreeChunks& p, hipStream_t st) {
  constexpr int COLS = 16 * CT * CW, KW = 4 / CW, TK = 32 * steps_of<HD, CT, CW>();
  constexpr int TILES = KW * (CW == 1 ? 1 : 2) * 2 * TK * HD * 2, JOIN = KW > 1 ? KW * COLS * (HD + SM_PAD) * 4 : 0, SMEM = TILES > JOIN ? TILES : JOIN;
  static std::atomic<uint64_t> lds_allowed{0};
  allow_dynamic_lds((const void*)k_tree_mfma<HD, CT, CW>, SMEM, lds_allowed);
  const int blocks = (a.max_nodes * (a.hq / a.hkv) + COLS - 1) / COLS;
  k_tree_mfma<HD, CT, CW><<<dim3(p.n, a.hkv * blocks, a.batch), 256, SMEM, st>>>(
      a.cu, a.seq_lens, a.parents, (const bf16*)a.qkv, a.cs, (bf16*)a.kc, (bf16*)a.vc, (bf16*)a.out, a.rows, a.hq, a.hkv, a.max_seq, p.n, p.keys / TK,
      p.o, p.ml);
  if (p.n > 1)
    k_tree_merge<HD><<<dim3(a.max_nodes, a.batch, (a.hq + 1024 / HD - 1) / (1024 / HD)), 256, 0, st>>>(a.cu, a.seq_lens, a.rows, a.hq, a.max_seq, p.n, p.keys,
                                                                                                   p.o, p.ml, (bf16*)a.out);
}

template <int HD>
void launch_hd(const TreeAttn& a, const TreeChunks& p, hipStream_t st) {
  const int cols = a.max_nodes * (a.hq / a.hkv);
  if (cols <= 16) launch<HD, 1, 1>(a, p, st);
  else if (cols <= 32) launch<HD, 1, 2>(a, p, st);
  else if (cols <= 64) launch<HD, 1, 4>(a, p, st);
  else launch<HD, 2, 4>(a, p, st);
}

}  // namespace

void launch_tree_attn_bf16(const TreeAttn& a, const TreeChunks& p, hipStream_t st) {
  if (a.hd == 128) launch_hd<128>(a, p, st);
  else launch_hd<64>(a, p, st);
}

}  // namespace ls
