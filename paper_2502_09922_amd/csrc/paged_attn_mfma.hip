// Attention of one new token a sequence over a cache in pages, on the matrix cores (head_dim 64 and 128).
//
// The query heads of a kv head are the columns of both products:
//   S^T[key][column] = K Q^T        A = 16 key rows, B = 16 columns
//   O^T[dim][column] += V^T P^T     A = V^T, B = P^T
// with the operand layouts, the split of bf16 queries and weights into two parts and the softmax of the attention of draft trees
// (tree_attn_mfma.hip): a lane of a result holds column lane % 16 and rows 4 (lane / 16) + e.  An output is rounded to bf16, of which two parts hold
// more than enough; the weights that slots get are fp32 and go by the scores, and with them queries keep
// all of their bits, in three parts (of two, 2^-16 of a score would be lost; 13B, 32 sequences of 500 slots, four layers 256.4 -> 257.8 us, 7B, 8 of 1024
// 124.7 -> 127.4).
//
// A workgroup is a (sequence, kv head, block of 16 columns, piece of the slots); its wavefronts take the piece's tiles in turn, each through a ring of
// LDS of its own that is filled straight from memory, so there are no barriers and what is on its way needs no registers: bound by memory, what
// counts is how many bytes a CU has asked for.  A page's number is a scalar (pages have at least eight slots, a wavefront's load covers
// eight rows at most) that is fetched a tile ahead.  The wavefronts' results are joined through LDS, those of pieces by a second
// kernel, both in order.
//
// The new token's row is put into its tile in LDS by the wavefront that has that tile, and into the cache: nobody waits for memory there.
//
// Bound by memory: 13B, 32 sequences of 1024 to 1087 slots (694 MB of cache) 107 us, 6.5 TB/s; with no arithmetic at all, the tiles only waited for,
// 106; the arithmetic alone 45.  70B, 64 of 128 to 2287 slots (366 MB) 60 us, 6.1 TB/s (66 when a CU's two workgroups were of the same sequence).  4 of
// 20001 to 32768 80, of which 5 are the second launch.  fp32, 13B, 16 of 1000 108, 6.0 TB/s, where a tile's products take half of its time on a
// SIMD.  Weights: where a workgroup has all of a sequence's slots, scores wait in LDS as far as there is room (13B, 32 sequences 121 us), otherwise they
// go out and come back, 4 bytes for each query head and slot: 70B, 64 others of 128 to 2287 slots (337 MB) 75 us instead of 56 (12 for the stores, 5 of
// which they cost where all of them go to the same lines; behind the fills or in another layout no less).
#include "attn_mfma.hpp"
#include "paged.hpp"

#include <algorithm>
#include <type_traits>

namespace ls {

namespace {

constexpr int SM_PAD = 4;          // floats behind a column's output in LDS: 16 columns' equal dims in different banks
constexpr int ORDERED = 256;       // sequences at most that are taken by length, whose lengths a wavefront holds in registers
constexpr int ORDERED_KEYS = 512;  // and only where some may be longer
constexpr float FOLLOW = 8.f;
constexpr int CUS = 256;
constexpr int TILE_KEYS = 16;  // as many rows as a matrix product has

__device__ __forceinline__ int wave_total(int v) {
  return __builtin_amdgcn_readfirstlane(
      __float_as_int(exchange<32, 1>(__int_as_float(v), [](float a, float b) { return __int_as_float(__float_as_int(a) + __float_as_int(b)); })));
}

// What workgroup `w` of `share` has to do where contexts are cut by their lengths: piece z of `pieces` of sequence b, for one of its `units` (kv heads x
// blocks of columns).  Pieces have at most `most` tiles, few enough of them that there are no more than `share` pieces; every wavefront finds that on
// its own, which takes a microsecond for 64 sequences.  False: nothing.
struct Piece {
  int b, unit, z, pieces, first;  // first: workgroup of the sequence's first piece
};
template <int C>
__device__ __forceinline__ bool deal(const PageMap& map, int batch, int units, int share, int w, int limit, int tile, Piece& p) {
  const int lane = threadIdx.x & 63;
  int tiles[C], total = 0;
#pragma unroll
  for (int c = 0; c < C; ++c) {  // a sequence without room has one, whose rows hold zeros
    const int i = c * 64 + lane, n = map.lens[min(i, batch - 1)];
    tiles[c] = i >= batch ? 0 : n < 0 || n >= limit || n >> map.shift >= map.columns ? 1 : n / tile + 1;
    total += tiles[c];
  }
  unsigned most = (unsigned)((wave_total(total) * (int64_t)units + share - 1) / share);
  int count[C];
  while (true) {
    int all = 0;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      count[c] = (int)(((unsigned)tiles[c] + most - 1) / most);
      all += count[c];
    }
    all = wave_total(all) * units;  // one for each sequence and unit in the end, for which there is room
    if (all <= share) break;
    most = max(most + 1, (unsigned)((uint64_t)most * (unsigned)all / (unsigned)share));
  }
  int before = 0;
  bool found = false;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    int upto = count[c];
    for (int off = 1; off < 64; off <<= 1) {
      const int v = __shfl_up(upto, off);
      upto += lane >= off ? v : 0;
    }
    const int first = (before + upto - count[c]) * units;
    const uint64_t is = __builtin_amdgcn_ballot_w64(w >= first && w < first + count[c] * units);
    if (is) {
      const int at = __builtin_ctzll(is);
      p.b = c * 64 + at;
      p.first = __builtin_amdgcn_readlane(first, at);
      p.pieces = __builtin_amdgcn_readlane(count[c], at);
      found = true;
    }
    before += __builtin_amdgcn_readlane(upto, 63);
  }
  if (!found) return false;
  p.unit = (w - p.first) / p.pieces;
  p.z = (w - p.first) % p.pieces;
  return true;
}

// NW: wavefronts; NB: tiles of a ring, a power of two.  Weights: scores wait for the end in memory, or in LDS, behind the rings.
enum Weigh { NO_WEIGHTS = 0, IN_MEMORY = 1, IN_LDS = 2 };
template <class T, int HD, int NW, int NB, Weigh WEIGH>
__global__ void __launch_bounds__(64 * NW, 2)
k_paged_mfma(PageMap map, const T* __restrict__ qkv, const float* __restrict__ cs, T* __restrict__ kc, T* __restrict__ vc, int32_t* __restrict__ places,
             T* __restrict__ out, int hq, int hkv, int max_pos, int most, int half, int batch, PagedPieces p, float* __restrict__ weights) {
  constexpr int THREADS = 64 * NW, TK = TILE_KEYS;
  constexpr int ROWB = HD * sizeof(T), EPC = 16 / sizeof(T);
  constexpr int CPR = HD / EPC;    // 16-byte chunks of a row
  constexpr int RPI = 64 / CPR;    // rows that a wavefront's load covers
  constexpr int NL = TK / RPI;     // loads of a tile's keys, as many of its values
  constexpr int UNITS = TK / 8;    // parts of a tile that lie in one page whatever the page's size
  constexpr int TILE = TK * ROWB;
  constexpr int DT = HD / 16;
  constexpr bool APART = NB == 1;  // the next tile's keys are asked for as soon as this one's are read: fp32, 13B, 16 of 1000 slots 116 -> 108 us (bf16, two tiles, 106 -> 108)
  constexpr int STORES = WEIGH == IN_MEMORY ? 1 : 0;  // of a tile's scores
  static_assert(RPI <= 8 && (NB & (NB - 1)) == 0, "");
  typedef T T4 __attribute__((ext_vector_type(4)));
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];

  const int G = hq / hkv, blocks = (G + 15) / 16;
  int b = blockIdx.y, unit = blockIdx.x, z = blockIdx.z, len_of_b;
  Piece dealt{};
  if (p.share) {
    const bool any = batch <= 64 ? deal<1>(map, batch, hkv * blocks, p.share, blockIdx.x, most, TK, dealt)
                     : batch <= 256 ? deal<4>(map, batch, hkv * blocks, p.share, blockIdx.x, most, TK, dealt)
                                    : deal<PagedPieces::SEQUENCES / 64>(map, batch, hkv * blocks, p.share, blockIdx.x, most, TK, dealt);
    if (!any) return;
    b = dealt.b;
    unit = dealt.unit;
    z = dealt.z;
    if (unit == 0 && z == 0 && threadIdx.x == 0) p.dealt[b] = int2{dealt.first, dealt.pieces};
  }
  unit = __builtin_amdgcn_readfirstlane(unit);
  z = __builtin_amdgcn_readfirstlane(z);
  const int kh = unit / blocks, cb = unit % blocks, cols = min(16, G - cb * 16);
  // by length: the longest first, and where all workgroups fit the chip at once, two to a CU, the shortest beside the longest (a sequence's
  // heads are neighbours: the second half of the workgroups goes to the CUs where the first half is)
  if (half) {
    const int rank = b < half ? b : batch - 1 - (b - half);
    b = batch <= 64 ? row_by_length<1, true>(map.lens, batch, rank, 1 << 24, len_of_b) : row_by_length<ORDERED / 64, true>(map.lens, batch, rank, 1 << 24, len_of_b);
  }
  b = __builtin_amdgcn_readfirstlane(b);
  const int lane = threadIdx.x & 63, lr = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const size_t row0 = (size_t)b * hq + kh * G + cb * 16;  // output row of column 0
  // Nothing in the launch writes lengths, positions and table: scalar loads, which do not queue behind the tiles on their way.  The
  // first tile's pages and the queries are asked for before the length is known.
  typedef const __attribute__((address_space(4))) int32_t fixed;
  PagedSeq t;
  t.n = ((fixed*)(uintptr_t)map.lens)[b];
  t.pos = map.positions ? ((fixed*)(uintptr_t)map.positions)[b] : t.n;
  fixed* entries = (fixed*)(uintptr_t)(map.table + (size_t)b * map.columns);
  const int mask = (1 << map.shift) - 1;
  int t_lo = z * (p.keys / TK);
  if (p.share && t.n >= 0) t_lo = __builtin_amdgcn_readfirstlane((t.n / TK + 1) * z / dealt.pieces);  // as even as may be (2^20 tiles, 2^10 pieces at most)
  int page[UNITS];  // of the tile that is filled next
  auto look_up = [&](int i) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < UNITS; ++u) page[u] = entries[min(((t_lo + wave + i * NW) * TK + 8 * u) >> map.shift, map.columns - 1)];
  };
  look_up(0);
  constexpr int KS = sizeof(T) == 2 ? HD / 32 : HD / 16;  // reads of a row
  const T* rows = qkv + (size_t)b * (hq + 2 * hkv) * HD;
  const T* q = rows + (size_t)(kh * G + cb * 16 + min(lr, cols - 1)) * HD;  // columns behind the last are its copies
  u32x4 raw[KS];
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) raw[kk] = *reinterpret_cast<const u32x4*>(q + (kk * 4 + lg) * EPC);
  auto no_room = [&] {  // the rows hold zeros
    if (z == 0)
      for (int i = threadIdx.x; i < cols * HD; i += THREADS) out[row0 * HD + i] = from_f<T>(0.f);
  };
  if (t.n < 0 || t.n >= most || t.n >> map.shift >= map.columns || t.pos < 0 || (cs && t.pos >= max_pos)) {
    no_room();
    return;
  }
  t.page = entries[t.n >> map.shift];
  const int keys = t.n + 1, ntile = (keys + TK - 1) / TK;
  if (t_lo >= ntile) return;
  int t_hi = z == p.n - 1 ? ntile : min(t_lo + p.keys / TK, ntile);  // the last piece takes what is left
  if (p.share) t_hi = __builtin_amdgcn_readfirstlane(ntile * (z + 1) / dealt.pieces);
  const int count = max(0, (t_hi - t_lo - wave + NW - 1) / NW);    // tiles of this wavefront: t_lo + wave, NW further each time
  const int lrow = lane / CPR, lchunk = lane % CPR;

  // ---- the ring
  unsigned koff[NL], voff[NL];  // a row's piece from the first of its eight rows
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int r = i * RPI + lrow;
    koff[i] = (r & 7) * ROWB + ((lchunk ^ key_swizzle<T, HD>(r)) << 4);
    voff[i] = (r & 7) * ROWB + ((lchunk ^ value_swizzle<T, HD>(r)) << 4);
  }
  const unsigned lds0 = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem + wave * (NB * 2 * TILE);
  int next = 0;                 // tiles that have been asked for
  uint64_t gone = 0;            // whose parts have no page: UNITS bits for each of the last tiles asked for
  // Written in assembly: of the builtin the compiler knows that it writes LDS but not where, and would wait for the fills on their way
  // before it reads what has arrived.  (m0 is reserved, of which the compiler warns.)
  const T* vt_next[UNITS];  // values of the tile whose keys have been asked for last
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  auto piece = [](auto once, const T* base, unsigned off, unsigned to) __attribute__((always_inline)) {
    if constexpr (decltype(once)::value) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(to), "v"(off), "s"(base) : "memory", "m0");
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory", "m0");
  };
#pragma clang diagnostic pop
  // What one block of columns reads once does not stay in L2: 13B, 32 sequences 120 -> 106 us, 70B, 64 ragged 76 -> 66, by now 60 (32 heads over one,
  // 64 sequences of 2000 slots, which two blocks read: 21 and 24).
  auto rows_of_tile = [&](const T* const* from, const unsigned* off, unsigned to) __attribute__((always_inline)) {
    auto all = [&](auto once) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NL; ++i) piece(once, from[i * RPI / 8], off[i], to + i * 1024);
    };
    if (blocks == 1) all(std::true_type{});
    else all(std::false_type{});
  };
  auto fill_keys = [&]() __attribute__((always_inline)) {
    const int key0 = (t_lo + wave + next * NW) * TK;
    const T* kt[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u) {
      const int at = key0 + 8 * u;
      const bool there = (unsigned)page[u] < (unsigned)map.pages;  // others read some page, and count as not seen
      gone = gone << 1 | (at <= t.n && !there);
      const size_t row = page_row0(there ? page[u] : 0, hkv, kh, map.shift) + (at & mask);
      kt[u] = kc + row * HD;
      vt_next[u] = vc + row * HD;
    }
    rows_of_tile(kt, koff, lds0 + (next & (NB - 1)) * (2 * TILE));
  };
  auto fill_values = [&]() __attribute__((always_inline)) {
    rows_of_tile(vt_next, voff, lds0 + (next & (NB - 1)) * (2 * TILE) + TILE);
    ++next;
    look_up(next);
  };
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) asm volatile("" : "+v"(raw[kk]));  // waited for here, not behind the tiles
  while (next < min(count, NB)) {
    fill_keys();
    fill_values();
  }

  // ---- queries: this wavefront's 16 columns, turned
  const float* turn = cs + (size_t)t.pos * HD;
  f32x4 angles[KS][EPC / 4];
#pragma unroll
  for (int kk = 0; kk < KS; ++kk)
#pragma unroll
    for (int e = 0; e < EPC / 4; ++e) angles[kk][e] = cs ? reinterpret_cast<const f32x4*>(turn + (kk * 4 + lg) * EPC)[e] : f32x4{1.f, 0.f, 1.f, 0.f};
  // the new token's row, a 16-byte piece to a lane: keys, and values behind them
  const bool mine = count > 0 && t_lo + wave + (count - 1) * NW == ntile - 1;
  const int nc = lane % CPR;
  const bool nv = lane >= CPR;
  u32x4 fresh{};
  f32x4 nturn[EPC / 4] = {};
  if (mine) {
    fresh = *reinterpret_cast<const u32x4*>(rows + (size_t)(hq + (nv ? hkv : 0) + kh) * HD + nc * EPC);
    if (cs)
#pragma unroll
      for (int e = 0; e < EPC / 4; ++e) nturn[e] = reinterpret_cast<const f32x4*>(turn + nc * EPC)[e];
  }
  if ((unsigned)t.page >= (unsigned)map.pages) {
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));  // nothing is on its way into the LDS of whoever comes next
    no_room();
    return;
  }

  // bf16: queries in two parts, in three where slots' weights go by the scores too
  constexpr int PARTS = sizeof(T) == 4 ? 1 : WEIGH ? 3 : 2;
  typedef std::conditional_t<sizeof(T) == 2, bf16x8, f32x4> Q;
  Q qp[PARTS][KS];
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) {
    const Q u = __builtin_bit_cast(Q, raw[kk]);
    float w[EPC];
#pragma unroll
    for (int e = 0; e < EPC; ++e) w[e] = to_f(u[e]);
    if (cs)
#pragma unroll
      for (int e = 0; e < EPC; e += 2) {
        const float2 c2{angles[kk][e / 4][e % 4], angles[kk][e / 4][e % 4 + 1]};
        const float w0 = turn0(w[e], w[e + 1], c2), w1 = turn1(w[e], w[e + 1], c2);
        w[e] = w0;
        w[e + 1] = w1;
      }
#pragma unroll
    for (int e = 0; e < EPC; ++e) {
      if constexpr (sizeof(T) == 2) {
        bf16 part[PARTS];
        if constexpr (WEIGH) three_parts(w[e], part);
        else two_parts(w[e], part[0], part[1]);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) qp[p][kk][e] = part[p];
      } else {
        qp[0][kk][e] = w[e];
      }
    }
  }
  if (mine) {
    if (cs && !nv) {
      Q u = __builtin_bit_cast(Q, fresh);
#pragma unroll
      for (int e = 0; e < EPC; e += 2) {
        const float2 c2{nturn[e / 4][e % 4], nturn[e / 4][e % 4 + 1]};
        const float u0 = to_f(u[e]), u1 = to_f(u[e + 1]);
        u[e] = from_f<T>(turn0(u0, u1, c2));
        u[e + 1] = from_f<T>(turn1(u0, u1, c2));
      }
      fresh = __builtin_bit_cast(u32x4, u);
    }
    if (cb == 0) {  // of blocks of columns one writes it
      const size_t slot = page_row0(t.page, hkv, kh, map.shift) + (t.n & mask);
      if (lane < 2 * CPR) *reinterpret_cast<u32x4*>((nv ? vc : kc) + slot * HD + nc * EPC) = fresh;
      if (WEIGH && lane == 0) places[slot] = t.pos;
    }
  }

  // Slots whose weights this thread adds up below, AHEAD at a time: where they are, and what they have, on its way while tiles are (at the end they
  // would be waited for: 13B, 32 sequences of 500 slots 65 us).
  constexpr int AHEAD = 4;
  size_t to[AHEAD];
  float had[AHEAD];
  bool there[AHEAD];
  auto weights_of = [&](int first) {
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int slot = min(first + j * THREADS, t.n), at = map.table[(size_t)b * map.columns + (slot >> map.shift)];
      there[j] = (unsigned)at < (unsigned)map.pages;
      to[j] = page_row0(there[j] ? at : 0, hkv, kh, map.shift) + (slot & mask);
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) had[j] = weights[to[j]];
  };
  if (WEIGH && weights) weights_of(threadIdx.x);
  float* scores = WEIGH == IN_MEMORY ? p.scores + (row0 + lr) * p.stride : nullptr;  // of this lane's column
  float* sm_s = reinterpret_cast<float*>(smem + NW * NB * 2 * TILE);

  // Sums of NEAR tiles are added to those of all tiles in front: one tile after the other, equal weights next to a long sum are all rounded the same
  // way (fp32, 2048 tiles of a wavefront: outputs off by 4.8e-4 of themselves, so 6e-6; 13B, 32 sequences 106.9 -> 107.4 us).
  constexpr int NEAR = 16;
  f32x4 o[DT], far_o[DT];
  float m_run = -INFINITY, l_run = 0.f, far_l = 0.f;  // l_run: of this lane's keys
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = far_o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  const float scale = 1.4426950408889634f / sqrtf((float)HD);  // q k -> exponent of 2
  // four neighbouring dims that a lane holds of a column: i of DT such, from dim_of(i) on
  auto dim_of = [&](int i) { return sizeof(T) == 2 ? i * 16 + 4 * lg : (i >> 2) * 64 + 16 * lg + 4 * (i & 3); };
  auto out_at = [&](int i, int e) -> float& {
    float* at = reinterpret_cast<float*>(&o[0]);
    return sizeof(T) == 2 ? at[i * 4 + e] : at[((i & ~3) + e) * 4 + (i & 3)];
  };

  for (int i = 0; i < count; ++i) {
    const int key0 = (t_lo + wave + i * NW) * TK;
    unsigned char* ks = smem + wave * (NB * 2 * TILE) + (i & (NB - 1)) * (2 * TILE);
    unsigned char* vs = ks + TILE;
    // Tile i has landed: behind its fills are those of the tiles asked for since, and the stores of the scores since then.  In a ring of one tile
    // its keys have, behind whose fills are its values'.
    const bool more = next < count;
    if constexpr (APART) wait_vm(NL + min(i, 1) * STORES);
    else if (next - i == NB && i >= NB - 1) __builtin_amdgcn_s_waitcnt(waitcnt_vm((NB - 1) * (2 * NL + STORES)));
    else wait_vm((next - 1 - i) * 2 * NL + min(i, NB - 1) * STORES);
    asm volatile("" ::: "memory");
    const unsigned units = (unsigned)(gone >> ((next - 1 - i) * UNITS)) & ((1u << UNITS) - 1);  // the highest bit is the first part's
    const bool masked = units || key0 + TK > keys, last = mine && i == count - 1;
    unsigned seen = (1u << TK) - 1;
    if (masked) {
#pragma unroll
      for (int u = 0; u < UNITS; ++u)
        if (units >> (UNITS - 1 - u) & 1) seen &= ~(0xFFu << (8 * u));
      if (key0 + TK > keys) seen &= (1u << (keys - key0)) - 1;
    }
    const int new_row = t.n - key0;
    if (last) {
      if (lane < CPR) *reinterpret_cast<u32x4*>(ks + new_row * ROWB + ((nc ^ key_swizzle<T, HD>(new_row)) << 4)) = fresh;
      asm volatile("" ::: "memory");
    }

    // ---- scores: all of a tile's keys are asked for at once, and all of its values before the softmax
    f32x4 s{0.f, 0.f, 0.f, 0.f};
    Q kf[KS];
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) kf[kk] = *reinterpret_cast<const Q*>(ks + lr * ROWB + (((kk * 4 + lg) ^ key_swizzle<T, HD>(lr)) << 4));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int part = PARTS - 1; part >= 0; --part) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[kk], qp[part][kk], s, 0, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[kk][e], qp[0][kk][e], s, 0, 0, 0);
      }
    }
    if constexpr (APART) {
      if (more) {  // over this tile's keys, of which every read has its value by now
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        fill_keys();
      }
      wait_vm(more ? NL : 0);  // its values
      asm volatile("" ::: "memory");
    }
    if (masked || last) {
      // values that nobody sees may be anything: zero times that has to be zero
#pragma unroll
      for (int j = 0; j < NL; ++j)
        if (!(seen >> (j * RPI + lrow) & 1)) *reinterpret_cast<u32x4*>(vs + j * 1024 + lane * 16) = u32x4{0u, 0u, 0u, 0u};
      if (last && nv && lane < 2 * CPR) *reinterpret_cast<u32x4*>(vs + new_row * ROWB + ((nc ^ value_swizzle<T, HD>(new_row)) << 4)) = fresh;
      asm volatile("" ::: "memory");
    }
    // bf16: the k index of the second product runs over keys {4g..4g+3}, g = lane / 16, fp32: row 4g + e, dims 16-byte chunk by chunk
    s16x4 vt[sizeof(T) == 2 ? DT : 1];
    Q vf[sizeof(T) == 2 ? 1 : DT];
    if constexpr (sizeof(T) == 2) {
      const int k0 = 4 * lg + (lr >> 2), within = (lr & 1) * 8;  // of the 16-byte chunk that holds dims 4 (lr % 4) of 16
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const int ch = d * 2 + ((lr & 3) >> 1);
        vt[d] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vs + k0 * ROWB + ((ch ^ value_swizzle<T, HD>(k0)) << 4) + within));
      }
    } else {
#pragma unroll
      for (int j = 0; j < HD / 64; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) vf[j * 4 + e] = *reinterpret_cast<const Q*>(vs + (4 * lg + e) * ROWB + (j * 16 + lr) * 16);
    }
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (WEIGH != NO_WEIGHTS) {
      if (lr < cols) *reinterpret_cast<f32x4*>((WEIGH == IN_LDS ? sm_s + lr * p.held : scores) + key0 + 4 * lg) = s;
    }
    if (masked) {
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] = seen >> (4 * lg + j) & 1u ? s[j] : -INFINITY;
    }
    // ---- softmax.  A NaN score makes its weight NaN, and the sums with it, whatever the maximum is.
    float mx = s[0];
#pragma unroll
    for (int j = 1; j < 4; ++j) mx = __builtin_elementwise_maximum(mx, s[j]);
    // The reference of the exponentials follows a maximum that has moved by more than 2^FOLLOW only: weights above one are as exact as below.
    auto far = [&] { return (mx - m_run) * scale > FOLLOW; };  // false for (-inf, -inf)
    if (__builtin_amdgcn_ballot_w64(far()) != 0) {             // lanes of a column exchange their maxima only then
      mx = exchange<16, 32>(mx, Max{});
      const bool moved = far();  // the others keep their bits
      const float m_new = fmaxf(m_run, mx);
      const float corr = moved ? __builtin_amdgcn_exp2f((m_run - m_new) * scale) : 1.f;
      l_run *= corr;
      far_l *= corr;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        o[d] *= corr;
        far_o[d] *= corr;
      }
      m_run = moved ? m_new : m_run;
    }
    const float mc = m_run == -INFINITY ? 0.f : m_run * scale;
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] = __builtin_amdgcn_exp2f(fmaf(s[j], scale, -mc));
    l_run += (s[0] + s[1]) + (s[2] + s[3]);
    // ---- output
    if constexpr (sizeof(T) == 2) {
      bf16x4 pf[2];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16 first, second;
        two_parts(s[j], first, second);
        pf[0][j] = first;
        pf[1][j] = second;
      }
#pragma unroll
      for (int part = 1; part >= 0; --part)
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vt[d], __builtin_bit_cast(s16x4, pf[part]), o[d], 0, 0, 0);
    } else {
#pragma unroll
      for (int j = 0; j < HD / 64; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int d = 0; d < 4; ++d) o[j * 4 + d] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[j * 4 + e][d], s[e], o[j * 4 + d], 0, 0, 0);
    }
    if (i % NEAR == NEAR - 1) {
      far_l += l_run;
      l_run = 0.f;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        far_o[d] += o[d];
        o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    }
    if (more) {  // over this tile, of which every read has its value by now
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if constexpr (!APART) fill_keys();
      fill_values();
    }
  }

  // ---- the wavefronts' results, in their order
  l_run = exchange<16, 32>(l_run + far_l, Add{});
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] += far_o[d];
  __shared__ float sm_m[NW][16], sm_l[NW][16];
  __shared__ float2 sm_all[16];  // maximum, 1 / sum
  __syncthreads();  // nobody reads tiles any more
  float* sm_o = reinterpret_cast<float*>(smem);
  if (lg == 0) {
    sm_m[wave][lr] = m_run;
    sm_l[wave][lr] = l_run;
  }
  if (lr < cols)
#pragma unroll
    for (int i = 0; i < DT; ++i)
      *reinterpret_cast<f32x4*>(sm_o + (wave * 16 + lr) * (HD + SM_PAD) + dim_of(i)) = f32x4{out_at(i, 0), out_at(i, 1), out_at(i, 2), out_at(i, 3)};
  __syncthreads();
  const bool whole = p.share ? dealt.pieces == 1 : ntile <= p.keys / TK || p.n == 1;  // the sequence is this one piece: its output rows go out
  const size_t place0 = p.share ? (size_t)blockIdx.x * 16 : (size_t)z * batch * hq + row0;
  for (int i = threadIdx.x; i < cols * (HD / 4); i += THREADS) {
    const int c = i / (HD / 4), d = i % (HD / 4) * 4;
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, sm_m[w][c]);
    f32x4 num{0.f, 0.f, 0.f, 0.f};
    float den = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      // sums without a maximum are zeros, or no numbers
      const float mw = sm_m[w][c], wt = mw == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((mw - m) * scale);
      const f32x4 v = *reinterpret_cast<const f32x4*>(sm_o + (w * 16 + c) * (HD + SM_PAD) + d);
#pragma unroll
      for (int e = 0; e < 4; ++e) num[e] += v[e] * wt;
      den += sm_l[w][c] * wt;
    }
    const size_t row = row0 + c;
    if (whole) {
      T4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = from_f<T>(num[e] / den);
      *reinterpret_cast<T4*>(out + row * HD + d) = v;
    } else {
      *reinterpret_cast<f32x4*>(p.o + (place0 + c) * HD + d) = num;
    }
    if (d == 0) {
      if (WEIGH && weights) sm_all[c] = float2{m == -INFINITY ? 0.f : m, 1.f / den};
      else if (WEIGH || !whole) p.ml[place0 + c] = float2{m, den};
    }
  }
  if constexpr (WEIGH != NO_WEIGHTS) {  // the weights of all slots, where one workgroup has all of them and all of the query heads
    if (!weights) return;
    __syncthreads();  // the scores of all wavefronts are in memory
    for (int first = threadIdx.x; first < keys; first += AHEAD * THREADS) {
      constexpr int U = 4;  // heads on their way at once
      float got[AHEAD] = {};
      for (int c0 = 0; c0 < cols; c0 += U) {
        float v[U][AHEAD];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int j = 0; j < AHEAD; ++j) {
            const int c = min(c0 + u, cols - 1), slot = min(first + j * THREADS, t.n);
            v[u][j] = WEIGH == IN_LDS ? sm_s[c * p.held + slot] : p.scores[(row0 + c) * p.stride + slot];
          }
        if (c0 == 0 && first != (int)threadIdx.x) weights_of(first);  // behind the scores, which wait for nothing
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (c0 + u < cols)
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) got[j] += __builtin_amdgcn_exp2f((v[u][j] - sm_all[c0 + u].x) * scale) * sm_all[c0 + u].y;
      }
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int slot = first + j * THREADS;
        if (slot < keys && there[j]) weights[to[j]] = slot == t.n ? got[j] : had[j] + got[j];
      }
    }
  }
}

// Bytes of scores that fit beside the rings without taking a place on the CU from another workgroup.
template <int NW> constexpr int HELD = NW == 4 ? 13 << 10 : 28 << 10;

template <class T, int HD, int NW, int NB, Weigh WEIGH>
void launch_kernel_of(const PagedAttn& a, const PagedPieces& p, int most, hipStream_t st) {
  constexpr int TILES = NW * NB * 2 * TILE_KEYS * HD * (int)sizeof(T), JOIN = NW * 16 * (HD + SM_PAD) * 4;
  static_assert(TILES >= JOIN && TILES <= NW * 16384, "");
  static std::atomic<uint64_t> lds_allowed{0};
  auto kernel = k_paged_mfma<T, HD, NW, NB, WEIGH>;
  allow_dynamic_lds((const void*)kernel, TILES + (WEIGH == IN_LDS ? HELD<NW> : 0), lds_allowed);
  const unsigned lds = TILES + (WEIGH == IN_LDS ? a.hq / a.hkv * p.held * 4 : 0);
  const int heads = a.hkv * ((a.hq / a.hkv + 15) / 16);
  int half = 0;
  if (p.n == 1 && !p.share && a.batch > 1 && a.batch <= ORDERED && a.max_keys > ORDERED_KEYS) half = (long)heads * a.batch <= 2 * CUS ? std::max(1, CUS / heads) : a.batch;
  kernel<<<p.share ? dim3(p.share) : dim3(heads, a.batch, p.n), 64 * NW, lds, st>>>(a.map, (const T*)a.qkv, a.cs, (T*)a.kc, (T*)a.vc, a.places, (T*)a.out, a.hq, a.hkv, a.max_pos, most, half,
                                                           a.batch, p, paged_joins_weights(a, p) ? a.weights : nullptr);
}

// Four wavefronts with two tiles each, two workgroups to a CU (fp32 of 128 dims: one tile of 16 KB), or twice the wavefronts where a CU has one
// workgroup at most.  13B, 32 sequences 106 us when these were compared; three wavefronts 110, two 116, tiles of 32 keys or rings of four tiles, which leave a CU one
// workgroup, 7 to 8 more.  7B, 8 sequences of 1024 slots with weights: eight wavefronts 27.0, four 29.1 (28.1 since queries have three parts).
// Scores of one workgroup that has all of a sequence's slots stay in LDS where they fit: 13B, 32 sequences of 1024 to 1087 slots 121 us, 132 through memory.
template <class T, int HD, int NW, int NB>
void launch_nw(const PagedAttn& a, PagedPieces p, int most, hipStream_t st) {
  p.held = p.stride + 4;  // columns' equal slots in different banks
  if (!a.weights) launch_kernel_of<T, HD, NW, NB, NO_WEIGHTS>(a, p, most, st);
  else if (paged_joins_weights(a, p) && (int64_t)(a.hq / a.hkv) * p.held * 4 <= HELD<NW>) launch_kernel_of<T, HD, NW, NB, IN_LDS>(a, p, most, st);
  else launch_kernel_of<T, HD, NW, NB, IN_MEMORY>(a, p, most, st);
}
template <class T, int HD>
void launch_hd(const PagedAttn& a, const PagedPieces& p, int most, hipStream_t st) {
  constexpr int NB = sizeof(T) * HD == 512 ? 1 : 2;
  const bool alone = (p.share ? p.share : (long)a.batch * a.hkv * ((a.hq / a.hkv + 15) / 16) * p.n) <= CUS;
  if (alone) launch_nw<T, HD, 8, NB>(a, p, most, st);
  else launch_nw<T, HD, 4, NB>(a, p, most, st);
}

}  // namespace

// Whether the attention kernel adds the weights up itself.
bool paged_joins_weights(const PagedAttn& a, const PagedPieces& p) { return a.weights && p.n == 1 && !p.share && a.hq / a.hkv <= 16; }

void launch_paged_attn_mfma(uint32_t dt, const PagedAttn& a, const PagedPieces& p, int most, hipStream_t st) {
  if (dt == F32) {
    if (a.hd == 128) launch_hd<float, 128>(a, p, most, st);
    else launch_hd<float, 64>(a, p, most, st);
  } else {
    if (a.hd == 128) launch_hd<bf16, 128>(a, p, most, st);
    else launch_hd<bf16, 64>(a, p, most, st);
  }
}

}  // namespace ls
