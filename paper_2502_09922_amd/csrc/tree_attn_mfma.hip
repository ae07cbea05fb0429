// Attention of draft trees on the matrix cores (head_dim 64 and 128).
//
// Nodes x query heads of a kv head are the columns of both products, all of which see the cached keys:
//   S^T[key][column] = K Q^T        A = 16 key rows, B = 16 columns
//   O^T[dim][column] += V^T P^T     A = V^T, B = P^T
// A lane of a result holds column lane % 16 and rows 4 (lane / 16) + e: one column's running maximum and sum are per-lane values
// and exchanges with lanes +-16 and +-32, and the weights that a lane has are a B operand as they are.
//   bf16: v_mfma_f32_16x16x32_bf16, steps of 32 keys.  The k index of the second product runs over keys {4g..4g+3, 16+4g..16+4g+3},
// g = lane / 16; V^T comes out of transposing LDS reads of the row-major tile.  Queries are turned in fp32; they and the weights enter as sums
// of two bf16 (two_parts): rounded once, queries would move every score by 2^-9 of its size, which costs more than the rounding of the
// output, and weights outputs by as much as that (70B, 64 ragged trees 89 us with one part of the weights, 101 with two; fewer columns wait for
// memory).  The parts are of one sign and the second is never zero, so that infinite keys and values are what they are in one product.
//   fp32: v_mfma_f32_16x16x4_f32, steps of 16 keys.  The k index is lane / 16; a 16-byte read of a key's or a value's row serves four
// products, of dims 16 j + 4 g + e of a key, and of rows 64 j + 4 (lane % 16) + e of V^T, which are the dims that a result's
// lane holds 4 apart.
//
// A workgroup is a (sequence, kv head, block of columns, chunk of keys).  Of its four wavefronts CW share keys, each with columns
// of its own, and 4 / CW split the chunk's keys.  Up to 16 columns each walks keys of its own, a tile at a time through registers into LDS of
// its own, no barriers (CW = 1); wavefronts that share keys fill a ring of tiles together, straight from memory, one barrier a tile.
// The splits' results are joined through LDS, chunks' by a second kernel, both in order.
//
// The nodes' own rows are turned, rounded and written to their slots by whoever reads those, a wavefront (CW = 1) or a workgroup,
// before it reads them: blocks of columns write the same bytes, and none depends on another workgroup's.  Only in the tiles of
// those slots columns see different keys.
//
// Bound by memory where columns are few: 13B, 32 sequences of 1024 to 1087 keys, 16 nodes (723 MB of cache) 130 us, 5.5 TB/s.  With
// many columns a tile's chain of reads, products, softmax and products is waited for, with two or three wavefronts on a SIMD: 70B, 64
// trees of 4 to 16 nodes over 128 to 2287 keys (128 columns) 97 to 101 us, the matrix cores busy for 35 % of it, the vector
// units for 38 %, LDS for 18 %, no bank conflicts; the longest context has 72 tiles, and 44 are the average of the places for workgroups.
// One sequence waits for its preamble (bounds, parents, table, queries:
// 5 us) and the second launch (4 us): 7B, 3000 keys, 26 nodes 19 us of which 7 are the cache's reading.
#include "tree.hpp"

#include <algorithm>
#include <type_traits>

namespace ls {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// 16-byte chunks of a row of a tile are permuted by its key, so that 16 rows' equal chunks (keys) and 4 rows' 32 bytes (values,
// transposing) lie in different banks.
template <class T, int HD> __device__ __forceinline__ int key_swizzle(int key) { return HD == 128 || sizeof(T) == 4 ? key & 15 : ((key & 3) << 1) | ((key >> 2) & 1); }
template <class T, int HD> __device__ __forceinline__ int value_swizzle(int key) {
  return sizeof(T) == 4 ? 0 : HD == 128 ? (key & 7) << 1 : ((key & 3) << 1) | ((key >> 2) & 1);
}

// v as a sum of two bf16: the first is v cut off, the second the rest, rounded, at least 2^-23 of v and of its sign.  Off by 2^-15 of v at
// most; infinite factors take part with their sign alone (inf + 0 inf or inf - inf would be no number).  0 stays 0.
__device__ __forceinline__ void two_parts(float v, bf16& first, bf16& second) {
  const unsigned bits = __builtin_bit_cast(unsigned, v);
  first = __builtin_bit_cast(bf16, (unsigned short)(bits >> 16));
  second = (bf16)fmaf(v, 0x1.000002p0f, -__builtin_bit_cast(float, bits & 0xFFFF0000u));
}

// Values that are no numbers become zeros; whether there were any.
template <class T>
__device__ __forceinline__ bool drop_nonfinite(u32x4& v) {
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      const bool bad = (v[i] & 0x7F800000u) == 0x7F800000u;
      any |= bad;
      v[i] = bad ? 0u : v[i];
    } else {
      const bool lo = (v[i] & 0x7F80u) == 0x7F80u, hi = (v[i] & 0x7F800000u) == 0x7F800000u;
      any |= lo || hi;
      v[i] &= (lo ? 0u : 0xFFFFu) | (hi ? 0u : 0xFFFF0000u);
    }
  }
  return any;
}

// A 16-byte piece of a row from dim `at` on, turned by its position's table row.
__device__ __forceinline__ u32x4 turned(u32x4 v, const float* turn, bf16) {
  const bf16x8 u = __builtin_bit_cast(bf16x8, v);
  const f32x4 ta = reinterpret_cast<const f32x4*>(turn)[0], tb = reinterpret_cast<const f32x4*>(turn)[1];
  bf16x8 w;
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const float2 c2 = p < 2 ? float2{ta[2 * p], ta[2 * p + 1]} : float2{tb[2 * p - 4], tb[2 * p - 3]};
    w[2 * p] = (bf16)turn0((float)u[2 * p], (float)u[2 * p + 1], c2);
    w[2 * p + 1] = (bf16)turn1((float)u[2 * p], (float)u[2 * p + 1], c2);
  }
  return __builtin_bit_cast(u32x4, w);
}
__device__ __forceinline__ u32x4 turned(u32x4 v, const float* turn, float) {
  const f32x4 u = __builtin_bit_cast(f32x4, v), c = *reinterpret_cast<const f32x4*>(turn);
  f32x4 w;
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    w[2 * p] = turn0(u[2 * p], u[2 * p + 1], float2{c[2 * p], c[2 * p + 1]});
    w[2 * p + 1] = turn1(u[2 * p], u[2 * p + 1], float2{c[2 * p], c[2 * p + 1]});
  }
  return __builtin_bit_cast(u32x4, w);
}

constexpr int SM_PAD = 4;  // floats behind a column's output in LDS: 16 columns' equal dims in different banks

constexpr int ORDERED = 256;       // sequences whose lengths a wavefront holds in registers
constexpr int ORDERED_KEYS = 512;  // contexts are ordered only where some may be longer
constexpr float FOLLOW = 8.f;
constexpr int CUS = 256;
// CW = 4 lives with two tiles and 168 registers, so that three workgroups fit a CU: 13B, 16 trees of 64 nodes over 1000 keys 89 us (90 since
// weights have two parts), with two (four tiles, 170 registers) 96; fp32, 4 such trees 82 either way.  CW = 2 in 168 registers gains nothing (148 and 151 us of kernel for 13B, 32
// x 26 nodes): its tiles leave room for two.
template <int CW> constexpr int PER_CU = CW == 4 ? 3 : 2;  // workgroups on a CU, wavefronts on a SIMD
template <class T> constexpr int TILE_KEYS = sizeof(T) == 2 ? 32 : 16;  // 16 KB of keys and values of 128 dims

// NB: tiles of the ring, a power of two (CW > 1).  Four instead of two, where LDS had room, changed nothing but what fits a CU.
template <class T, int HD, int CW, int KW, int NB>
__global__ void __launch_bounds__(64 * CW * KW, PER_CU<CW>)
k_tree_mfma(const int32_t* __restrict__ cu, const int32_t* __restrict__ seq_lens, const int32_t* __restrict__ parents, const T* __restrict__ qkv,
            const float* __restrict__ cs, T* __restrict__ kc, T* __restrict__ vc, T* __restrict__ out, int rows, int most, int hq, int hkv, int max_seq,
            int nchunk, int chunk_tiles, int half, float* __restrict__ part_o, float2* __restrict__ part_ml) {
  constexpr int THREADS = 64 * CW * KW;
  constexpr int TK = TILE_KEYS<T>;
  constexpr int ROWB = HD * sizeof(T), EPC = 16 / sizeof(T);
  constexpr int CPR = HD / EPC;          // 16-byte chunks of a row
  constexpr int RPI = 64 / CPR;          // rows that a wavefront's load covers
  constexpr int NL = TK / RPI / CW;      // loads of a wavefront for a tile's keys, as many for its values
  constexpr int TILE = TK * ROWB;
  constexpr int COLS = 16 * CW;  // of a workgroup
  constexpr int DT = HD / 16;
  typedef T T4 __attribute__((ext_vector_type(4)));
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];

  const int G = hq / hkv;
  const int kh = blockIdx.y % hkv, cb = blockIdx.y / hkv, z = blockIdx.x;
  int b = blockIdx.z, pos_of_b;
  // by length: the longest first, and where all workgroups fit the chip at once, two to a CU, the shortest beside the longest
  // (70B, 64 ragged trees take 88 us instead of 110; equal lengths pay for it: 13B, 16 trees of 64 nodes 88.2 and 86.5)
  if (half) {
    const int rank = b < half ? b : (int)gridDim.z - 1 - (b - half);
    b = gridDim.z <= 64 ? row_by_length<1, true>(seq_lens, gridDim.z, rank, max_seq, pos_of_b)
                        : row_by_length<ORDERED / 64, true>(seq_lens, gridDim.z, rank, max_seq, pos_of_b);
  }
  b = __builtin_amdgcn_readfirstlane(b);
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  TreeSeq t;
  const bool room = tree_seq(cu, seq_lens, b, rows, most, max_seq, t);
  if (cb * COLS >= t.n * G) return;
  if (!room) {  // the rows hold zeros
    if (z == 0 && cb == 0)
      for (int i = threadIdx.x; i < t.n * G * HD; i += THREADS) {
        const int c = i / HD;
        out[((size_t)(t.row0 + c / G) * hq + kh * G + c % G) * HD + i % HD] = from_f<T>(0.f);
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
  T *kb = kc + head0, *vb = vc + head0;
  const int stride = (hq + 2 * hkv) * HD;
  const T* rows0 = qkv + (size_t)t.row0 * stride;
  const int lrow = lane / CPR, lchunk = lane % CPR;
  const int first_row = share * NL * RPI;  // of a tile, that this wavefront brings

  u32x4 kreg[NL], vreg[NL];
  auto load = [&](int tile) {  // rows' byte offsets are of 32 bits behind the tile's address
    const int row0 = tile * TK + first_row;
    const char *kt = (const char*)(kb + (size_t)row0 * HD), *vt = (const char*)(vb + (size_t)row0 * HD);
    auto fetch = [&](int i, int from) {
      const int r = first_row + i * RPI + lrow;
      const u32x4* kp = reinterpret_cast<const u32x4*>(kt + from * ROWB + (unsigned)((lchunk ^ key_swizzle<T, HD>(r)) << 4));
      const u32x4* vp = reinterpret_cast<const u32x4*>(vt + from * ROWB + (unsigned)((lchunk ^ value_swizzle<T, HD>(r)) << 4));
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
  // CW > 1: straight into the ring.  Written in assembly: of the builtin the compiler knows that it writes LDS but not where, and would
  // wait for the fills on their way before it reads what has arrived.  (m0 is reserved, of which the compiler warns.)
  const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem + split * (NB * 2 * TILE) + first_row * ROWB;
  unsigned koff[NL], voff[NL];  // a row's piece from the tile's first row
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int r = first_row + i * RPI + lrow;
    koff[i] = r * ROWB + ((lchunk ^ key_swizzle<T, HD>(r)) << 4);
    voff[i] = r * ROWB + ((lchunk ^ value_swizzle<T, HD>(r)) << 4);
  }
  auto fill = [&](int tile) {
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
    auto piece = [](const T* base, unsigned off, unsigned to) {
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory", "m0");
    };
#pragma clang diagnostic pop
    const T *kt = kb + (size_t)tile * TK * HD, *vt = vb + (size_t)tile * TK * HD;
    const unsigned to = lds0 + ((tile - t_begin) & (NB - 1)) * (2 * TILE);
    const int have = keys - tile * TK;
    if (have >= TK) {
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        piece(kt, koff[i], to + i * 1024);
        piece(vt, voff[i], to + TILE + i * 1024);
      }
    } else {  // rows behind the last key: that one again, which their weights of zero leave out
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int r = first_row + i * RPI + lrow;
        const unsigned back = (unsigned)(r - min(r, have - 1)) * ROWB;
        piece(kt, koff[i] - back, to + i * 1024);
        piece(vt, voff[i] - back, to + TILE + i * 1024);
      }
    }
  };
  // on their way while nodes and queries are made ready: tiles without nodes
  bool early = false;
  int next = t_begin;  // the next tile to be filled
  if constexpr (CW == 1) {
    early = t_begin < t_end && (t_begin + 1) * TK <= t.ctx;
    if (early) load(t_begin);
  } else {
    while (next < min(t_end, t_begin + NB - 1) && (next + 1) * TK <= t.ctx) fill(next++);
  }

  // this wavefront's 16 columns
  constexpr int KS = sizeof(T) == 2 ? HD / 32 : HD / 16;  // reads of a row
  const int col = cb * COLS + share * 16 + lr;
  const bool busy = cb * COLS + share * 16 < t.n * G, in = col < t.n * G;
  const int node = in ? col / G : 0;
  const T* q = rows0 + (size_t)node * stride + (size_t)(kh * G + (in ? col % G : 0)) * HD;
  u32x4 raw[KS];
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) raw[kk] = *reinterpret_cast<const u32x4*>(q + (kk * 4 + lg) * EPC);
  const uint64_t path = tree_path(parents, t);
  {  // the nodes' rows among the keys of this wavefront (CW = 1) or workgroup
    const int depth = __builtin_popcountll(path) - 1;
    const int n_lo = max((CW == 1 ? t_begin : t_lo) * TK, t.ctx), items = (min((CW == 1 ? t_end : t_hi) * TK, keys) - n_lo) * CPR;
    constexpr int STEP = CW == 1 ? 64 : THREADS;
    for (int i0 = 0; i0 < items; i0 += STEP) {
      const int i = i0 + (CW == 1 ? lane : (int)threadIdx.x), key = n_lo + i / CPR, ch = i % CPR, j = min(key - t.ctx, t.n - 1);
      const int d = __shfl(depth, j);
      if (i < items) {
        const T* row = rows0 + (size_t)j * stride + ch * EPC;
        u32x4 k = *reinterpret_cast<const u32x4*>(row + (size_t)(hq + kh) * HD);
        const u32x4 v = *reinterpret_cast<const u32x4*>(row + (size_t)(hq + hkv + kh) * HD);
        if (cs) k = turned(k, cs + (size_t)(t.ctx + d) * HD + ch * EPC, T{});
        *reinterpret_cast<u32x4*>(kb + (size_t)key * HD + ch * EPC) = k;
        *reinterpret_cast<u32x4*>(vb + (size_t)key * HD + ch * EPC) = v;
      }
    }
    if (items > 0) {  // other lanes of this wavefront read them, or of the workgroup
      if constexpr (CW == 1) __threadfence_block();
      else __syncthreads();
    }
  }

  // ---- queries, bf16 as two parts, and the nodes they see
  typedef std::conditional_t<sizeof(T) == 2, bf16x8, f32x4> Q;
  Q qh[KS], ql[sizeof(T) == 2 ? KS : 1];
  const uint64_t sees = (uint64_t)(unsigned)__shfl((int)(unsigned)(path >> 32), node) << 32 | (unsigned)__shfl((int)(unsigned)path, node);
  const float* turn = cs + (size_t)(t.ctx + __builtin_popcountll(sees) - 1) * HD;
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) {
    const int d0 = (kk * 4 + lg) * EPC;
    if constexpr (sizeof(T) == 4) {
      qh[kk] = __builtin_bit_cast(f32x4, cs ? turned(raw[kk], turn + d0, T{}) : raw[kk]);
    } else {
      const bf16x8 u = __builtin_bit_cast(bf16x8, raw[kk]);
      f32x4 ta{}, tb{};
      if (cs) {
        ta = reinterpret_cast<const f32x4*>(turn + d0)[0];
        tb = reinterpret_cast<const f32x4*>(turn + d0)[1];
      }
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        float u0 = (float)u[2 * p], u1 = (float)u[2 * p + 1];
        if (cs) {
          const float2 c2 = p < 2 ? float2{ta[2 * p], ta[2 * p + 1]} : float2{tb[2 * p - 4], tb[2 * p - 3]};
          const float w0 = turn0(u0, u1, c2), w1 = turn1(u0, u1, c2);
          u0 = w0;
          u1 = w1;
        }
        bf16 first[2], second[2];
        two_parts(u0, first[0], second[0]);
        two_parts(u1, first[1], second[1]);
        qh[kk][2 * p] = first[0];
        qh[kk][2 * p + 1] = first[1];
        ql[kk][2 * p] = second[0];
        ql[kk][2 * p + 1] = second[1];
      }
    }
  }

  f32x4 o[DT];
  float m_run = -INFINITY;
  float l_run = 0.f;  // of this lane's keys
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float scale = 1.4426950408889634f / sqrtf((float)HD);  // score -> exponent of 2
  // four neighbouring dims that a lane holds of a column: i of DT such, from dim_of(i) on
  auto dim_of = [&](int i) { return sizeof(T) == 2 ? i * 16 + 4 * lg : (i >> 2) * 64 + 16 * lg + 4 * (i & 3); };
  auto out_at = [&](int i, int e) -> float& {
    float* at = reinterpret_cast<float*>(&o[0]);
    return sizeof(T) == 2 ? at[i * 4 + e] : at[((i & ~3) + e) * 4 + (i & 3)];
  };
  auto piece = [&](int i) { return f32x4{out_at(i, 0), out_at(i, 1), out_at(i, 2), out_at(i, 3)}; };

  // ---- a tile in LDS
  constexpr int HALVES = TK / 16;
  auto attend = [&](const unsigned char* ks, const unsigned char* vs, int key0, bool odd) {
    f32x4 s[HALVES];
    // all of a tile's keys are asked for at once, and all of its values before the softmax: with a few reads at a time each of them
    // was waited for
    Q kf[HALVES][KS];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
      const int kl = h * 16 + lr;
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) kf[h][kk] = *reinterpret_cast<const Q*>(ks + kl * ROWB + (((kk * 4 + lg) ^ key_swizzle<T, HD>(kl)) << 4));
      s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
          for (int h = 0; h < HALVES; ++h) s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[h][kk], part ? qh[kk] : ql[kk], s[h], 0, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) s[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[0][kk][e], qh[kk][e], s[0], 0, 0, 0);
      }
    }
    Q vt[DT];  // bf16: 16 dims each; fp32: a read of four, of which there are as many
    if constexpr (sizeof(T) == 2) {
      const int k0 = 4 * lg + (lr >> 2), k1 = k0 + 16;
      const int within = (lr & 1) * 8;  // of the 16-byte chunk that holds dims 4 (lr % 4) of 16
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const int ch = d * 2 + ((lr & 3) >> 1);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vs + k0 * ROWB + ((ch ^ value_swizzle<T, HD>(k0)) << 4) + within));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vs + k1 * ROWB + ((ch ^ value_swizzle<T, HD>(k1)) << 4) + within));
        vt[d] = __builtin_bit_cast(Q, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      }
    } else {
#pragma unroll
      for (int j = 0; j < HD / 64; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) vt[j * 4 + e] = *reinterpret_cast<const Q*>(vs + (4 * lg + e) * ROWB + (j * 16 + lr) * 16);
    }
    __builtin_amdgcn_sched_barrier(0);
    const int behind = key0 - t.ctx;  // of the cached positions
    if (behind > -TK) {               // slots of nodes
      const unsigned seen = behind >= 64 ? 0u : behind >= 0 ? (unsigned)(sees >> behind) : (unsigned)(sees << -behind) | ((1u << -behind) - 1u);
#pragma unroll
      for (int i = 0; i < 4 * HALVES; ++i) s[i >> 2][i & 3] = seen >> ((i >> 2) * 16 + 4 * lg + (i & 3)) & 1u ? s[i >> 2][i & 3] : -INFINITY;
    }
    // a NaN score makes its weight NaN, and the sums with it, whatever the maximum is
    float mx = s[0][0];
#pragma unroll
    for (int i = 1; i < 4 * HALVES; ++i) mx = __builtin_elementwise_maximum(mx, s[i >> 2][i & 3]);
    // The reference of the exponentials follows a maximum that has moved by more than 2^FOLLOW only: bf16 and fp32 weights above one
    // are as exact as below.  Following every move, and adding up the sums here, took 70B, 64 ragged trees 5 % longer.
    auto far = [&] { return (mx - m_run) * scale > FOLLOW; };  // false for (-inf, -inf)
    if (__builtin_amdgcn_ballot_w64(far()) != 0) {             // lanes of a column exchange their maxima only then
      mx = exchange<16, 32>(mx, Max{});
      const bool moved = far();  // the others keep their bits
      const float m_new = fmaxf(m_run, mx);
      const float corr = moved ? __builtin_amdgcn_exp2f((m_run - m_new) * scale) : 1.f;
      l_run *= corr;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= corr;
      m_run = moved ? m_new : m_run;
    }
    const float mc = m_run == -INFINITY ? 0.f : m_run * scale;
#pragma unroll
    for (int i = 0; i < 4 * HALVES; ++i) s[i >> 2][i & 3] = __builtin_amdgcn_exp2f(fmaf(s[i >> 2][i & 3], scale, -mc));
    // four products less of 68 in fp32; in bf16 (a row of ones) the registers for it are not there
    l_run += (s[0][0] + s[0][1]) + (s[0][2] + s[0][3]);
    if constexpr (sizeof(T) == 2) {
      l_run += (s[1][0] + s[1][1]) + (s[1][2] + s[1][3]);
      bf16x8 pf[2];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        bf16 first, second;
        two_parts(s[i >> 2][i & 3], first, second);
        pf[0][i] = first;
        pf[1][i] = second;
      }
#pragma unroll
      for (int part = 1; part >= 0; --part)
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt[d], pf[part], o[d], 0, 0, 0);
    } else {
#pragma unroll
      for (int j = 0; j < HD / 64; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int d = 0; d < 4; ++d) o[j * 4 + d] = __builtin_amdgcn_mfma_f32_16x16x4f32(vt[j * 4 + e][d], s[0][e], o[j * 4 + d], 0, 0, 0);
    }
    if (odd) {  // nodes' values that are no numbers lie in the tile as zeros: only the columns that see the nodes take them
      for (int j = max(0, -behind); j < TK && behind + j < t.n; ++j) {
        const T* v = rows0 + (size_t)(behind + j) * stride + (size_t)(hq + hkv + kh) * HD;
        float p = 0.f;
#pragma unroll
        for (int i = 0; i < 4 * HALVES; ++i) p = (j >> 4) * 4 + (j & 3) == i ? s[i >> 2][i & 3] : p;
        p = __shfl(p, ((j >> 2) & 3) * 16 + lr);
        if (!(sees >> (behind + j) & 1)) continue;
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          const T4 x = *reinterpret_cast<const T4*>(v + dim_of(i));
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!(fabsf(to_f(x[e])) < INFINITY)) out_at(i, e) += p * to_f(x[e]);
          __builtin_amdgcn_sched_barrier(0);  // rare: no registers for it
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
        if (tile * TK + first_row + i * RPI + lrow >= t.ctx) odd |= drop_nonfinite<T>(vreg[i]);
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

  __shared__ int odd_flags[NB][CW * KW];
  unsigned char* tiles = smem + split * ((CW == 1 ? 1 : NB) * 2 * TILE);
  if constexpr (CW > 1)
    while (next < min(t_end, t_begin + NB - 1)) fill(next++);
  if constexpr (CW == 1) {
    for (int i = t_begin - 1; i < t_end; ++i) {  // tile i is attended to while i + 1 is on its way
      bool odd = false;
      if (i >= t_begin) odd = put(tiles, tiles + TILE, i);
      if (i + 1 < t_end && (i >= t_begin || !early)) load(i + 1);
      if (i >= t_begin) attend(tiles, tiles + TILE, i * TK, odd);
    }
  } else {
    for (int i = t_begin; i < t_begin + per; ++i) {  // as many turns for all
      unsigned char* ks = tiles + ((i - t_begin) & (NB - 1)) * (2 * TILE);
      int* flags = odd_flags[(i - t_begin) & (NB - 1)];
      const bool last = (i + 1) * TK > t.ctx;  // slots of nodes
      if (i < t_end) {
        // this wavefront's fills of tile i have landed: those behind it are 2 NL for each tile
        if (next - i == NB - 1) __builtin_amdgcn_s_waitcnt(waitcnt_vm((NB - 2) * 2 * NL));
        else wait_vm((next - 1 - i) * 2 * NL);
        asm volatile("" ::: "memory");
        if (last) {  // as put() does, in what this wavefront has filled
          bool odd = false;
#pragma unroll
          for (int j = 0; j < NL; ++j) {
            const int r = first_row + j * RPI;
            u32x4* at = reinterpret_cast<u32x4*>(ks + TILE + r * ROWB + lane * 16);
            u32x4 v = *at;
            if (i * TK + r + lrow >= t.ctx && drop_nonfinite<T>(v)) {
              odd = true;
              *at = v;
            }
          }
          if (lane == 0) flags[wave] = 0;
          if (__builtin_amdgcn_ballot_w64(odd) != 0 && lane == 0) flags[wave] = 1;
        }
      }
      slot_barrier<true>();
      if (next < t_end) fill(next++);  // over tile i - 1, which all have left
      if (i < t_end && busy) {
        int odd = 0;
        if (last)
#pragma unroll
          for (int w = 0; w < CW; ++w) odd |= flags[split * CW + w];
        attend(ks, ks + TILE, i * TK, odd != 0);
      }
    }
  }

  l_run = exchange<16, 32>(l_run, Add{});
  if constexpr (KW > 1) {  // ---- the splits' results, in their order
    __shared__ float sm_m[KW][COLS], sm_l[KW][COLS];
    __syncthreads();  // nobody reads tiles any more
    float* sm_o = reinterpret_cast<float*>(smem);
    const int at = share * 16 + lr;
    if (lg == 0) {
      sm_m[split][at] = m_run;
      sm_l[split][at] = l_run;
    }
#pragma unroll
    for (int i = 0; i < DT; ++i) *reinterpret_cast<f32x4*>(sm_o + (split * COLS + at) * (HD + SM_PAD) + dim_of(i)) = piece(i);
    __syncthreads();
    for (int i = threadIdx.x; i < COLS * (HD / 4); i += THREADS) {
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
        T4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = from_f<T>(num[e] / den);
        *reinterpret_cast<T4*>(out + row * HD + d) = v;
      } else {
        *reinterpret_cast<f32x4*>(part_o + (pieces + row) * HD + d) = num;
        if (d == 0) part_ml[pieces + row] = float2{m, den};
      }
    }
  } else {
    int at = threadIdx.x;  // the column found again: it would hold a register through the loop
    asm volatile("" : "+v"(at));
    at = cb * COLS + share * 16 + (at & 15);
    if (at >= t.n * G) return;
    const size_t row = row_of(at);
    if (whole) {
      const float inv = 1.0f / l_run;
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        const f32x4 p = piece(i);
        T4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = from_f<T>(p[e] * inv);
        *reinterpret_cast<T4*>(out + row * HD + dim_of(i)) = v;
      }
    } else {
#pragma unroll
      for (int i = 0; i < DT; ++i) *reinterpret_cast<f32x4*>(part_o + (pieces + row) * HD + dim_of(i)) = piece(i);
      if (lg == 0) part_ml[pieces + row] = float2{m_run, l_run};
    }
  }
}

// Rows of sequences of several chunks: the chunks' results in chunk order, four dims to a thread.  They are asked for before it is known
// whose row this is, and how many of them there are.  Whose it is all sequences are asked: bounds that only the device knows need not rise.
template <class T, int HD>
__global__ void __launch_bounds__(256)
k_tree_merge(const float* __restrict__ part_o, const float2* __restrict__ part_ml, const int32_t* __restrict__ cu, const int32_t* __restrict__ seq_lens,
             int rows, int most, int hq, int batch, int max_seq, int nchunk, int chunk_keys, T* __restrict__ out) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  constexpr int TPR = HD / 4, U = 8;  // chunks on their way at once
  const int r = blockIdx.x, h = min((int)(blockIdx.y * (256 / TPR) + threadIdx.x / TPR), hq - 1), d = threadIdx.x % TPR * 4;
  const size_t row = (size_t)r * hq + h, step = (size_t)rows * hq;
  float2 ml[U];
  f32x4 v[U];
  auto load = [&](int z0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const size_t at = row + min(z0 + u, nchunk - 1) * step;
      ml[u] = part_ml[at];
      v[u] = *reinterpret_cast<const f32x4*>(part_o + at * HD + d);
    }
  };
  load(0);
  __shared__ int whose;
  if (threadIdx.x == 0) whose = batch;
  __syncthreads();
  TreeSeq t;
  for (int b = threadIdx.x; b < batch; b += 256)
    if (tree_seq(cu, seq_lens, b, rows, most, max_seq, t) && r >= t.row0 && r < t.row0 + t.n) atomicMin(&whose, b);
  __syncthreads();
  if (whose == batch) return;
  tree_seq(cu, seq_lens, whose, rows, most, max_seq, t);
  const int n = min((t.ctx + t.n + chunk_keys - 1) / chunk_keys, nchunk);
  if (n == 1) return;  // the first pass wrote these rows
  const float scale = 1.4426950408889634f / sqrtf((float)HD);
  float m = -INFINITY, den = 0.f;
  f32x4 num{0.f, 0.f, 0.f, 0.f};
  for (int z0 = 0; z0 < n; z0 += U) {
    if (z0) load(z0);
    float top = m;
#pragma unroll
    for (int u = 0; u < U; ++u) top = z0 + u < n ? fmaxf(top, ml[u].x) : top;
    const float corr = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * scale);
    den *= corr;
    num *= corr;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (z0 + u < n) {
        const float wt = ml[u].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((ml[u].x - top) * scale);
#pragma unroll
        for (int e = 0; e < 4; ++e) num[e] += v[u][e] * wt;
        den += ml[u].y * wt;
      }
    m = top;
  }
  T4 w;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = from_f<T>(num[e] / den);
  *reinterpret_cast<T4*>(out + row * HD + d) = w;
}

template <class T, int HD, int CW, int KW, int NB>
void launch(const TreeAttn& a, const TreeChunks& p, hipStream_t st) {
  constexpr int COLS = 16 * CW, TK = TILE_KEYS<T>;
  constexpr int TILES = KW * NB * 2 * TK * HD * (int)sizeof(T), JOIN = KW > 1 ? KW * COLS * (HD + SM_PAD) * 4 : 0;
  constexpr int SMEM = TILES > JOIN ? TILES : JOIN;
  static std::atomic<uint64_t> lds_allowed{0};
  allow_dynamic_lds((const void*)k_tree_mfma<T, HD, CW, KW, NB>, SMEM, lds_allowed);
  const int blocks = (a.max_nodes * (a.hq / a.hkv) + COLS - 1) / COLS;
  const long each = (long)a.hkv * blocks;  // workgroups of a sequence
  int half = 0;
  if (p.n == 1 && a.batch > 1 && a.batch <= ORDERED && a.max_keys > ORDERED_KEYS) half = each * a.batch <= PER_CU<CW> * CUS ? std::max(1, (int)(CUS / each)) : a.batch;
  k_tree_mfma<T, HD, CW, KW, NB><<<dim3(p.n, a.hkv * blocks, a.batch), 64 * CW * KW, SMEM, st>>>(
      a.cu, a.seq_lens, a.parents, (const T*)a.qkv, a.cs, (T*)a.kc, (T*)a.vc, (T*)a.out, a.rows, a.max_nodes, a.hq, a.hkv, a.max_seq, p.n, p.keys / TK, half, p.o, p.ml);
  if (p.n > 1)
    k_tree_merge<T, HD><<<dim3(a.rows, (a.hq + 1024 / HD - 1) / (1024 / HD)), 256, 0, st>>>(p.o, p.ml, a.cu, a.seq_lens, a.rows, a.max_nodes, a.hq, a.batch, a.max_seq,
                                                                                       p.n, p.keys, (T*)a.out);
}

// Wavefronts share keys where columns are too many for one, as few as do.  7B, one sequence of 3000 keys, 26 nodes: 18.5 us with two 16-
// column tiles in each pair of wavefronts, 23 with both in every wavefront, keys of its own.  Blocks of 64 columns at most, which read the cache
// again, four fifths of it out of L2: blocks of 128, two tiles to a wavefront and two workgroups to a CU, took 92 us instead of 88 for 70B, 64
// ragged trees, 58 instead of 53 for 16 of them, 34 instead of 30 for one of 64 nodes over 4000 keys (with weights of one part; the latter are
// 101, 58 and 33 now).
template <class T, int HD>
void launch_hd(const TreeAttn& a, const TreeChunks& p, hipStream_t st) {
  const int cols = a.max_nodes * (a.hq / a.hkv);
  if (cols <= 16) launch<T, HD, 1, 4, 1>(a, p, st);
  else if (cols <= 32) launch<T, HD, 2, 2, 2>(a, p, st);
  else launch<T, HD, 4, 1, 2>(a, p, st);
}

}  // namespace

void launch_tree_attn_mfma(uint32_t dt, const TreeAttn& a, const TreeChunks& p, hipStream_t st) {
  if (dt == F32) {
    if (a.hd == 128) launch_hd<float, 128>(a, p, st);
    else launch_hd<float, 64>(a, p, st);
  } else {
    if (a.hd == 128) launch_hd<bf16, 128>(a, p, st);
    else launch_hd<bf16, 64>(a, p, st);
  }
}

}  // namespace ls
