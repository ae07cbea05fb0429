// A cache in pages: the entry points of include/ls_stage.h, the filling of pages from a prompt pass's cache and the eviction of slots.
#include "entry.hpp"
#include "paged.hpp"

#include <algorithm>
#include <type_traits>


namespace ls {

namespace {

// ---- filling -----------------------------------------------------------------------------------------------------------------
constexpr int FILL_SLOTS = 64;  // a thread of a workgroup at most to each
struct FillArgs {
  PageMap map;
  const int32_t *src, *from_lens;
  int batch, from_batch, from_seq, hkv, heads, pieces, slots;  // heads: layer * hkv + kv head; pieces of a row
};

__device__ __forceinline__ int fill_len(const FillArgs& a, int b, int& src) {
  src = a.src[b];
  if ((unsigned)src >= (unsigned)a.from_batch) return -1;
  const int n = a.from_lens[src];
  return n <= a.from_seq && n <= a.slots ? n : -1;
}

// A workgroup to FILL_SLOTS slots of a (sequence, layer, kv head) at a time, a thread to a U-sized piece of a row, AT_ONCE of them on their way.
template <class U>
__global__ void __launch_bounds__(256)
k_paged_fill(FillArgs a, const U* __restrict__ fk, const U* __restrict__ fv, const float* __restrict__ fw, U* __restrict__ kc, U* __restrict__ vc,
             float* __restrict__ weights, int32_t* __restrict__ places, int32_t* __restrict__ lens, int32_t* __restrict__ positions, int blocks) {
  constexpr int AT_ONCE = 4;
  const int b = blockIdx.y, head = blockIdx.x / blocks, block = blockIdx.x % blocks, layer = head / a.hkv, kh = head % a.hkv;
  int src;
  const int n = fill_len(a, b, src);
  if (blockIdx.x == 0 && threadIdx.x == 0 && n >= 0) {  // nobody in this launch reads them
    lens[b] = n;
    if (positions) positions[b] = n;
  }
  const size_t from = (((size_t)layer * a.from_batch + src) * a.hkv + kh) * a.from_seq, layer0 = (size_t)layer * a.map.pages * a.hkv << a.map.shift;
  const int32_t* entries = a.map.table + (size_t)b * a.map.columns;
  auto row_of = [&](int slot, size_t& row) {
    const int page = entries[slot >> a.map.shift];
    row = layer0 + page_row0(page, a.hkv, kh, a.map.shift) + (slot & ((1 << a.map.shift) - 1));
    return (unsigned)page < (unsigned)a.map.pages;
  };
  for (int lo = block * FILL_SLOTS; lo < n; lo += blocks * FILL_SLOTS) {  // more than one only where max_len is understated
    const int slots = min(FILL_SLOTS, n - lo), items = slots * a.pieces;
    size_t place = 0;  // of a slot to a thread: its weight is on its way with the rows
    float weight = 0.f;
    const bool named = weights && (int)threadIdx.x < slots && row_of(lo + threadIdx.x, place);
    if (named && fw) weight = fw[from + lo + threadIdx.x];
    for (int i0 = threadIdx.x; i0 < items; i0 += 256 * AT_ONCE) {
      U k[AT_ONCE], v[AT_ONCE];
      size_t to[AT_ONCE];
      bool there[AT_ONCE];
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        const int i = min(i0 + j * 256, items - 1), slot = lo + i / a.pieces, piece = i % a.pieces;
        const size_t at = (from + slot) * a.pieces + piece;
        k[j] = __builtin_nontemporal_load(fk + at);
        v[j] = __builtin_nontemporal_load(fv + at);
        there[j] = row_of(slot, to[j]) && i0 + j * 256 < items;
        to[j] = to[j] * a.pieces + piece;
      }
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j)
        if (there[j]) {
          __builtin_nontemporal_store(k[j], kc + to[j]);
          __builtin_nontemporal_store(v[j], vc + to[j]);
        }
    }
    if (named) {
      weights[place] = weight;
      places[place] = lo + threadIdx.x;
    }
  }
}

// ---- eviction ----------------------------------------------------------------------------------------------------------------
struct EvictArgs {
  PageMap map;
  int batch, hkv, layers, keep, first, recent, max_len, most;  // most: moves of a (layer, sequence, kv head)
  float* weights;
  int32_t* places;
  int32_t* count;  // [units] moves that are to be made, -1 for a sequence that is left alone
  int2* moves;     // [units][most]: to slot x from slot y
  u32x4* keys;     // [units][wavefronts][groups / 4][64], where registers do not hold them
  int groups;      // of 64 slots to a wavefront, room for them
  void *kc, *vc;
  int pieces;      // of a row, 16 bytes each (wide) or 4
  bool wide;
};

// Greater keys stay.  A weight that is no number has 0, equal weights equal keys.
__device__ __forceinline__ unsigned stay_key(float w, int place, int first, int from) {
  if (place < first || place >= from) return 0xFFFFFFFFu;
  const unsigned bits = __builtin_bit_cast(unsigned, w + 0.f);  // -0 is 0
  return w != w ? 0u : bits ^ (bits >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}

__device__ __forceinline__ size_t slot_row(const EvictArgs& a, const int32_t* entries, int layer, int kh, int slot) {
  return page_row0(0, a.hkv, kh, a.map.shift) + (((size_t)layer * a.map.pages + entries[slot >> a.map.shift]) * a.hkv << a.map.shift) + (slot & ((1 << a.map.shift) - 1));
}

// Slots and positions of a unit's sequence; false if it is left alone, whose entries all threads of the workgroup look at.
__device__ __forceinline__ bool evict_seq(const EvictArgs& a, int b, int threads, int* bad, int& n, int& from) {
  n = a.map.lens[b];
  const int pos = a.map.positions[b];
  from = pos < a.recent ? 0 : pos - a.recent;
  if (n <= a.keep || n > a.max_len || (n - 1) >> a.map.shift >= a.map.columns) return false;
  const int32_t* entries = a.map.table + (size_t)b * a.map.columns;
  bool odd = false;
  for (int i = threadIdx.x; i <= (n - 1) >> a.map.shift; i += threads) odd |= (unsigned)entries[i] >= (unsigned)a.map.pages;
  if (threads == 64) return __builtin_amdgcn_ballot_w64(odd) == 0;
  if (threadIdx.x == 0) *bad = 0;
  __syncthreads();
  if (odd) *bad = 1;
  __syncthreads();
  return *bad == 0;
}

// `count` of the moves of a (layer, kv head), by `threads` threads: a U-sized piece of a row to each, AT_ONCE of them on their way.
template <class U>
__device__ __forceinline__ void make_moves(const EvictArgs& a, const int32_t* entries, int layer, int kh, const int2* moves, int count, int threads) {
  constexpr int AT_ONCE = 4;
  U *kc = (U*)a.kc, *vc = (U*)a.vc;
  const int items = count * a.pieces;
  for (int i0 = threadIdx.x; i0 < items; i0 += threads * AT_ONCE) {
    U k[AT_ONCE], v[AT_ONCE];
    size_t to[AT_ONCE];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int i = min(i0 + j * threads, items - 1), piece = i % a.pieces;
      const int2 m = moves[i / a.pieces];
      const size_t fr = slot_row(a, entries, layer, kh, m.y) * a.pieces + piece;
      to[j] = slot_row(a, entries, layer, kh, m.x) * a.pieces + piece;
      k[j] = __builtin_nontemporal_load(kc + fr);
      v[j] = __builtin_nontemporal_load(vc + fr);
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j)
      if (i0 + j * threads < items) {
        __builtin_nontemporal_store(k[j], kc + to[j]);
        __builtin_nontemporal_store(v[j], vc + to[j]);
      }
  }
  for (int i = threadIdx.x; i < count; i += threads) {
    const int2 m = moves[i];
    const size_t to = slot_row(a, entries, layer, kh, m.x), fr = slot_row(a, entries, layer, kh, m.y);
    a.weights[to] = a.weights[fr];
    a.places[to] = a.places[fr];
  }
}

constexpr int HELD = 1024 * 64;  // slots at most whose keys registers hold
// Rows of all kv heads of a layer, whose bytes of weights and places 32-bit offsets reach.
constexpr int64_t NARROW = 1 << 29;

// The moves of a (layer, sequence, kv head): W wavefronts, of which the w-th has the w-th part of the slots, 64 neighbours at a time.  The largest key that
// `keep` slots or more reach is searched for between the smallest and the largest of the slots that may go, by where it lay if keys were spread
// evenly, until exactly `keep` slots reach it or nothing is left between; in the latter case the lower ones of equal keys stay.  Weights and places
// are read once.  V > 0: the keys of up to 64 W V slots are held in V registers of a lane; V = 0: each lane leaves them in memory for itself, four of
// its slots side by side (8 units of 131072 slots 270 us, 930 when keys were made again for each count).
// Where a unit has no more than FEW moves (`here`), they are made here: another launch for one move each took 6 us for 5120 units.
// Bound by its steps one after the other: 70B, 128 units of up to 16384 slots down to 2048 26 us (16 wavefronts; 4 loads, 8 rounds, 4 list), 5120
// units of 501 slots, one move each, 15.
constexpr int FEW = 32, GUESSES = 12, GROUPS = 32;
template <int W, int V, class Row = unsigned>
__global__ void __launch_bounds__(64 * W) k_evict_choose(EvictArgs a, bool here) {
  constexpr int GR = 8, READ = GROUPS;  // keys at a time that are made, and that are read again; of no slot: 0, below every threshold
  const int unit = blockIdx.x, kh = unit % a.hkv, b = unit / a.hkv % a.batch, layer = unit / a.hkv / a.batch;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  __shared__ int bad, sums[2][W][3];
  __shared__ int2 list[FEW];
  int n, from, turn = 0;
  if (!evict_seq(a, b, 64 * W, &bad, n, from)) {
    if (threadIdx.x == 0) a.count[unit] = -1;
    return;
  }
  // over the workgroup: what each wavefront has, in order
  auto each = [&](int x, int y, int z) {
    turn ^= 1;
    if (lane == 0) {
      sums[turn][wave][0] = x;
      sums[turn][wave][1] = y;
      sums[turn][wave][2] = z;
    }
    __syncthreads();
  };
  __shared__ int counts[3];  // one is added to, one read, one cleared
  if (W > 1 && threadIdx.x == 0) counts[0] = 0;
  auto total = [&](int x, int round) {
    if constexpr (W == 1) return x;
    if (lane == 0) atomicAdd(&counts[round % 3], x);
    if (threadIdx.x == 0) counts[(round + 1) % 3] = 0;
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(counts[round % 3]);
  };
  const int32_t* entries = a.map.table + (size_t)b * a.map.columns;
  const int per = (n + 64 * W - 1) / (64 * W), first = wave * per * 64, slot0 = first + lane, mask = (1 << a.map.shift) - 1;
  const float* weights = a.weights + ((size_t)layer * a.map.pages * a.hkv << a.map.shift);
  const int32_t* places = a.places + ((size_t)layer * a.map.pages * a.hkv << a.map.shift);
  auto load = [&](int g, unsigned* k) __attribute__((always_inline)) {
    Row row[GR];
    float w[GR];
    int place[GR];
#pragma unroll
    for (int j = 0; j < GR; ++j) {
      const int slot = min(slot0 + (g + j) * 64, n - 1);
      row[j] = (((Row)entries[slot >> a.map.shift] * a.hkv + kh) << a.map.shift) + (slot & mask);
    }
#pragma unroll
    for (int j = 0; j < GR; ++j) {
      w[j] = weights[row[j]];
      place[j] = places[row[j]];
    }
#pragma unroll
    for (int j = 0; j < GR; ++j) k[j] = g + j < per && slot0 + (g + j) * 64 < n ? stay_key(w[j], place[j], a.first, from) : 0;
  };
  unsigned key[V > 0 ? V : READ];
  u32x4* mine = V > 0 ? nullptr : a.keys + ((size_t)unit * W + wave) * (a.groups / 4) * 64 + lane;
  if constexpr (V > 0) {
#pragma unroll
    for (int g = 0; g < V; g += GR) {
      if (g < per) {
        load(g, key + g);
      } else {
#pragma unroll
        for (int j = 0; j < GR; ++j) key[g + j] = 0;
      }
    }
  } else {
    for (int g = 0; g < per; g += READ) {
#pragma unroll
      for (int j = 0; j < READ; j += GR) load(g + j, key + j);
#pragma unroll
      for (int j = 0; j < READ; j += 4) mine[(g + j) / 4 * 64] = u32x4{key[j], key[j + 1], key[j + 2], key[j + 3]};
    }
  }
  // f(which of 64 slots, slot, key of it) over all slots of this wavefront and some behind, whose keys are 0
  auto all_slots = [&](auto f) __attribute__((always_inline)) {
    if constexpr (V > 0) {
#pragma unroll
      for (int g = 0; g < V; g += GR)
        if (g < per) {
#pragma unroll
          for (int i = g; i < g + GR; ++i) f(i, slot0 + i * 64, key[i]);
        }
    } else {
      for (int g = 0; g < per; g += READ) {
        u32x4 four[READ / 4];
#pragma unroll
        for (int j = 0; j < READ / 4; ++j) four[j] = mine[(g / 4 + j) * 64];
#pragma unroll
        for (int j = 0; j < READ; ++j) f(g + j, slot0 + (g + j) * 64, four[j / 4][j % 4]);
      }
    }
  };
  unsigned low = 0xFFFFFFFFu, high = 0;
  int stay = 0;  // slots that stay whatever their weight
  all_slots([&](int i, int slot, unsigned k) __attribute__((always_inline)) {
    const bool free = i < per && slot < n && k != 0xFFFFFFFFu;
    low = min(low, free ? k : 0xFFFFFFFFu);
    high = max(high, free ? k : 0u);
    stay += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k == 0xFFFFFFFFu));
  });
  auto bits = [](float v) { return __builtin_bit_cast(unsigned, v); };
  low = bits(exchange<32, 1>(__builtin_bit_cast(float, low), [&](float x, float y) { return __builtin_bit_cast(float, min(bits(x), bits(y))); }));
  high = bits(exchange<32, 1>(__builtin_bit_cast(float, high), [&](float x, float y) { return __builtin_bit_cast(float, max(bits(x), bits(y))); }));
  if constexpr (W > 1) {
    each((int)low, (int)high, stay);
    low = 0xFFFFFFFFu;
    high = stay = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      low = min(low, (unsigned)sums[turn][w][0]);
      high = max(high, (unsigned)sums[turn][w][1]);
      stay += sums[turn][w][2];
    }
  }
  low = __builtin_amdgcn_readfirstlane(low);
  high = __builtin_amdgcn_readfirstlane(high);
  // `reach` slots have at least `least`, `keep` or more of them; fewer than `keep`, `above`, have `beyond` or more
  unsigned least = low, beyond = high + 1;
  int reach = n, above = stay;
  if (stay >= a.keep) {
    least = 0xFFFFFFFFu;
    reach = stay;
    above = 0;
  }
  for (int round = 0; reach != a.keep && beyond - least > 1 && stay < a.keep; ++round) {
    const unsigned range = beyond - least;
    unsigned step = range >> 1;
    // 16384 weights spread like exp(1.5 N(0, 1)) take 8 rounds, by halves 14, in turn 13 to 16; halves end what guesses do not
    if (round < GUESSES) step = min(max((unsigned)((float)range * ((float)(reach - a.keep) / (float)(reach - above))), 1u), range - 1);
    const unsigned middle = __builtin_amdgcn_readfirstlane(least + step);
    int got = 0;
    all_slots([&](int, int, unsigned k) __attribute__((always_inline)) { got += __builtin_popcountll(__builtin_amdgcn_ballot_w64(k >= middle)); });
    got = total(got, round);
    if (got >= a.keep) {
      least = middle;
      reach = got;
    } else {
      beyond = middle;
      above = got;
    }
  }
  // ---- holes and movers in the order of slots
  const bool ties = reach != a.keep;  // of the slots of key `least`, keep - above stay
  int rank0 = 0;                      // of those, in front of this wavefront
  if (ties) {
    int equal = 0;
    all_slots([&](int i, int slot, unsigned k) __attribute__((always_inline)) { equal += __builtin_popcountll(__builtin_amdgcn_ballot_w64(i < per && slot < n && k == least)); });
    if constexpr (W > 1) {
      each(equal, 0, 0);
      for (int w = 0; w < wave; ++w) rank0 += sums[turn][w][0];
    }
  }
  auto before = [](uint64_t m) { return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0)); };  // lanes of m in front of this one
  auto stays = [&](int i, int slot, unsigned k, int& rank) __attribute__((always_inline)) {
    const bool there = i < per && slot < n;
    bool is = there && k >= least;
    if (ties) {
      const uint64_t equal = __builtin_amdgcn_ballot_w64(there && k == least);
      if (there && k == least) is = rank + before(equal) < a.keep - above;
      rank += __builtin_popcountll(equal);
    }
    return is;
  };
  int to = 0, fr = 0, all = 0;
  {
    int holes = 0, movers = 0, rank = rank0;
    all_slots([&](int i, int slot, unsigned k) __attribute__((always_inline)) {
      const uint64_t is = __builtin_amdgcn_ballot_w64(stays(i, slot, k, rank));
      const int64_t front = (int64_t)a.keep - (first + i * 64);  // of these 64 slots below `keep`
      const uint64_t in_front = i >= per || front <= 0 ? 0ull : front >= 64 ? ~0ull : (1ull << front) - 1;
      holes += __builtin_popcountll(~is & in_front);
      movers += __builtin_popcountll(is & ~in_front);
    });
    all = movers;
    if constexpr (W > 1) {
      each(holes, movers, 0);
      all = 0;
#pragma unroll
      for (int w = 0; w < W; ++w) {
        to += w < wave ? sums[turn][w][0] : 0;
        fr += w < wave ? sums[turn][w][1] : 0;
        all += sums[turn][w][1];
      }
    }
  }
  int2* moves = here ? list : a.moves + (size_t)unit * a.most;
  int rank = rank0;
  all_slots([&](int i, int slot, unsigned k) __attribute__((always_inline)) {
    const bool is = stays(i, slot, k, rank), hole = i < per && slot < a.keep && !is, mover = slot >= a.keep && is;
    const uint64_t hs = __builtin_amdgcn_ballot_w64(hole), ms = __builtin_amdgcn_ballot_w64(mover);
    if (hs) {
      if (hole) moves[to + before(hs)].x = slot;
      to += __builtin_popcountll(hs);
    }
    if (ms) {
      if (mover) moves[fr + before(ms)].y = slot;
      fr += __builtin_popcountll(ms);
    }
  });
  if (threadIdx.x == 0) a.count[unit] = here ? 0 : all;
  if (!here) return;
  __syncthreads();
  if (a.wide) make_moves<u32x4>(a, entries, layer, kh, list, all, 64 * W);
  else make_moves<uint32_t>(a, entries, layer, kh, list, all, 64 * W);
}

// The moves: a workgroup to MOVES of them at a time.  The lengths, which the launch before reads, are set by one workgroup of a sequence.
constexpr int MOVES = 64;
template <class U>
__global__ void __launch_bounds__(256) k_evict_move(EvictArgs a, int32_t* __restrict__ lens) {
  const int unit = blockIdx.x, kh = unit % a.hkv, b = unit / a.hkv % a.batch, layer = unit / a.hkv / a.batch;
  const int count = a.count[unit];
  if (count < 0) return;
  if (layer == 0 && kh == 0 && blockIdx.y == 0 && threadIdx.x == 0) lens[b] = a.keep;
  const int2* moves = a.moves + (size_t)unit * a.most;
  for (int lo = blockIdx.y * MOVES; lo < count; lo += gridDim.y * MOVES)
    make_moves<U>(a, a.map.table + (size_t)b * a.map.columns, layer, kh, moves + lo, min(MOVES, count - lo), 256);
}

// Lengths alone, where the moves have been made.
__global__ void __launch_bounds__(256) k_evict_lens(EvictArgs a, int32_t* __restrict__ lens) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  if (b < a.batch && a.count[b * a.hkv] >= 0) lens[b] = a.keep;
}

// Groups of 64 slots whose keys each of 16 wavefronts leaves in memory.
int key_groups(int max_len) { return max_len > HELD ? ((max_len + 1023) / 1024 + GROUPS - 1) / GROUPS * GROUPS : 0; }

void launch_evict(const EvictArgs& a, size_t units, int32_t* lens, hipStream_t st) {
  // As many registers as hold the keys, and more wavefronts to a unit where units do not fill the chip.  One slot to go, with the second launch, us:
  //    501 slots, 8 / 512 / 4096 units    one wavefront 12 / 18 / 18   four 17 / 22 / 38
  //   1025 slots, 64 / 2048 / 4096 units  one 25 / 26 / 31             four 16 / 27 / 36         sixteen 21 / 85 / 164
  //   2049 slots, 8 / 512 / 4096 units                                 four 15 / 26 / 53         sixteen 15 / 39 / 153
  //   4097 slots, 8 / 64 / 512 / 2048 units                            four 22 / 23 / 25 / 48    sixteen 18 / 20 / 29 / 82
  //   8000 slots, 8 / 64 / 512 units                                   four 25 / 25 / 30         sixteen 18 / 17 / 33
  // so that up to 512 slots one wavefront does, up to 4096 four; beyond, and below for one, it goes by the units.  (From 512 units on four would
  // do for 4097 to 8192 slots, which `few` leaves to sixteen.)
  const bool few = units <= 2048, here = a.most <= FEW;
  const int n = a.max_len;
  if (n > HELD) k_evict_choose<16, 0, size_t><<<units, 1024, 0, st>>>(a, here);
  else if (((int64_t)a.map.pages * a.hkv << a.map.shift) >= NARROW) k_evict_choose<16, 64, size_t><<<units, 1024, 0, st>>>(a, here);
  else if (n <= 64 * 8) k_evict_choose<1, 8><<<units, 64, 0, st>>>(a, here);
  else if (n <= 64 * 16 && !few) k_evict_choose<1, 16><<<units, 64, 0, st>>>(a, here);
  else if (n <= 64 * 32 && !few) k_evict_choose<1, 32><<<units, 64, 0, st>>>(a, here);
  else if (n <= 256 * 8) k_evict_choose<4, 8><<<units, 256, 0, st>>>(a, here);
  else if (n <= 256 * 16) k_evict_choose<4, 16><<<units, 256, 0, st>>>(a, here);
  else if (n <= 256 * 32 && !few) k_evict_choose<4, 32><<<units, 256, 0, st>>>(a, here);
  else if (n <= 1024 * 8) k_evict_choose<16, 8><<<units, 1024, 0, st>>>(a, here);
  else if (n <= 1024 * 16) k_evict_choose<16, 16><<<units, 1024, 0, st>>>(a, here);
  else if (n <= 1024 * 32) k_evict_choose<16, 32><<<units, 1024, 0, st>>>(a, here);
  else k_evict_choose<16, 64><<<units, 1024, 0, st>>>(a, here);
  if (here) {
    k_evict_lens<<<(a.batch + 255) / 256, 256, 0, st>>>(a, lens);
    return;
  }
  const dim3 grid(units, std::min((a.most + MOVES - 1) / MOVES, 1024));
  if (a.wide) k_evict_move<u32x4><<<grid, 256, 0, st>>>(a, lens);
  else k_evict_move<uint32_t><<<grid, 256, 0, st>>>(a, lens);
}

// ---- arguments ---------------------------------------------------------------------------------------------------------------
bool overlap(const void* a, uint64_t a_bytes, const void* b, uint64_t b_bytes) {
  return a && b && (uintptr_t)a < (uintptr_t)b + b_bytes && (uintptr_t)b < (uintptr_t)a + a_bytes;
}

const char* pages_error(const ls_heads* h, const ls_pages* p, int batch) {
  if (!p || !p->k || !p->v || !p->lens || !p->table) return "NULL ls_pages or pointer inside it";
  if (p->page < 8 || p->page > 1024 || (p->page & (p->page - 1))) return "page has to be a power of two from 8 to 1024";
  if (!p->pages || p->pages > (1u << 24)) return "pages outside [1, 2^24]";
  if (!p->columns || (uint64_t)p->columns * p->page > (1u << 24)) return "columns * page outside [1, 2^24]";
  if (!p->weights != !p->places) return "weights and places come together";
  if (batch < 1 || batch > (int)h->max_batch || batch > 65535) return "batch outside [1, max_batch], or beyond 65535";
  const uintptr_t size = h->dtype == LS_DTYPE_F32 ? 4 : 2;
  if (((uintptr_t)p->k | (uintptr_t)p->v) & (size - 1)) return "a pool is not aligned to its type";
  if (((uintptr_t)p->weights | (uintptr_t)p->places | (uintptr_t)p->lens | (uintptr_t)p->positions | (uintptr_t)p->table) & 3) return "a buffer is not aligned to its type";
  if (overlap(p->lens, h->max_batch * 4ull, p->positions, h->max_batch * 4ull)) return "lens and positions are one buffer";
  return nullptr;
}

// Whether no launch takes the weights of so many slots.
bool too_many_weights(const ls_heads* h, const ls_pages* p, int max_ctx) {
  return p->weights && (int64_t)h->n_kv_heads * ((int64_t)max_ctx / 256 + 1) >= (1 << 24) - (1 << 16);
}

PageMap map_of(const ls_pages* p) {
  PageMap m;
  m.lens = p->lens; m.positions = p->positions; m.table = p->table;
  m.pages = (int)p->pages; m.columns = (int)p->columns;
  while ((1u << m.shift) < p->page) ++m.shift;
  return m;
}

PagedAttn attn_of(const ls_heads* h, const ls_pages* p, int batch, int max_ctx) {
  PagedAttn a;
  a.map = map_of(p);
  a.kc = p->k; a.vc = p->v; a.weights = p->weights; a.places = p->places;
  a.batch = batch; a.hq = (int)h->n_q_heads; a.hkv = (int)h->n_kv_heads; a.hd = (int)h->head_dim; a.max_pos = (int)h->max_seq;
  a.size = h->dtype == LS_DTYPE_F32 ? 4 : 2; a.max_keys = max_ctx + 1;
  return a;
}

// The checks of an attention call that its sizing query shares; its bounds are in reach of LS_ERR_KV_OVERFLOW.
ls_status context_error(const char* who, const ls_heads* h, const ls_pages* p, int max_ctx, bool turns) {
  if (max_ctx < 0) return bad(who, "max_ctx is negative");
  if ((uint64_t)max_ctx + 1 > (uint64_t)p->columns * p->page) {
    set_last_error("%s: context %d + 1 exceeds the table's %u pages of %u", who, max_ctx, p->columns, p->page);
    return LS_ERR_KV_OVERFLOW;
  }
  if (turns && !p->positions && (uint64_t)max_ctx + 1 > h->max_seq) {
    set_last_error("%s: context %d + 1 exceeds max_seq %u", who, max_ctx, h->max_seq);
    return LS_ERR_KV_OVERFLOW;
  }
  return LS_OK;
}

}  // namespace

ls_status paged_attention_args(const char* who, const ls_heads* h, const ls_pages* p, int batch, int max_ctx, bool turns, void* scratch, size_t scratch_bytes,
                               PagedAttn* a) {
  if (const char* e = heads_error(h)) return bad(who, e);
  if (const char* e = pages_error(h, p, batch)) return bad(who, e);
  const ls_status rc = context_error(who, h, p, max_ctx, turns);
  if (rc != LS_OK) return rc;
  if (too_many_weights(h, p, max_ctx)) return bad(who, "weights of more slots than a launch takes");
  *a = attn_of(h, p, batch, max_ctx);
  if (a->weights) {
    const size_t need = paged_attn_scratch_bytes(*a);
    if (!scratch || scratch_bytes < need) {
      set_last_error("%s: %zu bytes of scratch, %zu are needed", who, scratch ? scratch_bytes : 0, need);
      return LS_ERR_OOM;
    }
    if ((uintptr_t)scratch & 15) return bad(who, "scratch is not aligned to 16 bytes");
  }
  a->scratch = ((uintptr_t)scratch & 15) ? nullptr : (float*)scratch;
  a->scratch_bytes = scratch_bytes;
  return LS_OK;
}

}  // namespace ls

namespace {

using ls::bad;
using ls::launched;

size_t evict_units(const ls_heads* h, int layers, int batch) { return (size_t)layers * batch * h->n_kv_heads; }

const char* evict_error(const ls_heads* h, int layers, int batch, int keep, int max_len) {
  if (const char* e = ls::heads_error(h)) return e;
  if (batch < 1 || batch > (int)h->max_batch || batch > 65535) return "batch outside [1, max_batch], or beyond 65535";
  if (layers < 1 || layers > (1 << 20) || evict_units(h, layers, batch) >= (1u << 22)) return "layers outside [1, what a launch takes]";
  if (keep < 1) return "keep has to be at least 1";
  if (max_len < 0 || max_len > (1 << 24)) return "max_len outside [0, 2^24]";
  return nullptr;
}

}  // namespace

extern "C" {

size_t ls_paged_attention_scratch_bytes(const ls_heads* h, const ls_pages* layer, int batch, int max_ctx) {
  if (ls::heads_error(h) || ls::pages_error(h, layer, batch) || max_ctx < 0 || (uint64_t)max_ctx + 1 > (uint64_t)layer->columns * layer->page || ls::too_many_weights(h, layer, max_ctx)) return 0;
  return ls::paged_attn_scratch_bytes(ls::attn_of(h, layer, batch, max_ctx));
}

ls_status ls_paged_attention(const ls_heads* h, const ls_pages* layer, int batch, int max_ctx, const void* qkv, const float* rope, void* out, void* scratch,
                             size_t scratch_bytes, void* hip_stream) {
  static const char* who = "ls_paged_attention";
  ls::PagedAttn a;
  const ls_status rc = ls::paged_attention_args(who, h, layer, batch, max_ctx, rope != nullptr, scratch, scratch_bytes, &a);
  if (rc != LS_OK) return rc;
  if (!qkv || !out) return bad(who, "NULL argument");
  const uintptr_t size = h->dtype == LS_DTYPE_F32 ? 4 : 2;
  if (((uintptr_t)qkv | (uintptr_t)out) & (size - 1)) return bad(who, "a buffer is not aligned to its type");
  if ((uintptr_t)rope & 7) return bad(who, "rope is not aligned to 8 bytes");
  const uint64_t row = (uint64_t)batch * h->head_dim * size;
  if (ls::overlap(qkv, row * (h->n_q_heads + 2ull * h->n_kv_heads), out, row * h->n_q_heads)) return bad(who, "out overlaps qkv");
  a.qkv = qkv; a.cs = rope; a.out = out;
  ls::launch_paged_attn(h->dtype, a, (hipStream_t)hip_stream);
  return launched(who);
}

ls_status ls_paged_fill(const ls_heads* h, int layers, const ls_kv* from, int from_batch, int from_seq, const int32_t* src, const float* weights, int max_len,
                        const ls_pages* pages, int batch, void* hip_stream) {
  static const char* who = "ls_paged_fill";
  if (const char* e = ls::heads_error(h)) return bad(who, e);
  if (const char* e = ls::pages_error(h, pages, batch)) return bad(who, e);
  if (!from || !from->k || !from->v || !from->seq_lens || !src) return bad(who, "NULL argument");
  if (from_batch < 1 || from_batch >= (1 << 24) || from_seq < 1 || from_seq > (1 << 24)) return bad(who, "from_batch outside [1, 2^24) or from_seq outside [1, 2^24]");
  const uintptr_t at = (uintptr_t)from->k | (uintptr_t)from->v | (uintptr_t)pages->k | (uintptr_t)pages->v;
  if (at & 3) return bad(who, "a cache is not aligned to 4 bytes");
  if (((uintptr_t)src | (uintptr_t)from->seq_lens | (uintptr_t)weights) & 3) return bad(who, "a buffer is not aligned to its type");
  if (ls::overlap(from->seq_lens, from_batch * 4ull, pages->lens, batch * 4ull) || ls::overlap(from->seq_lens, from_batch * 4ull, pages->positions, batch * 4ull))
    return bad(who, "seq_lens overlaps lens or positions");
  if (max_len < 0) return bad(who, "max_len is negative");
  const size_t row = (size_t)h->head_dim * (h->dtype == LS_DTYPE_F32 ? 4 : 2);
  const bool wide = row % 16 == 0 && (at & 15) == 0;
  ls::FillArgs a;
  a.map = ls::map_of(pages);
  a.src = src; a.from_lens = from->seq_lens; a.batch = batch; a.from_batch = from_batch; a.from_seq = from_seq;
  a.hkv = (int)h->n_kv_heads; a.pieces = (int)(row / (wide ? 16 : 4)); a.slots = (int)(pages->columns * pages->page);
  const int most = std::max(1, std::min({max_len, from_seq, a.slots})), blocks = (most + ls::FILL_SLOTS - 1) / ls::FILL_SLOTS;
  if (layers < 1 || (uint64_t)layers * h->n_kv_heads * blocks >= (1u << 24)) return bad(who, "layers outside [1, what a launch takes]");
  a.heads = layers * a.hkv;
  hipStream_t st = (hipStream_t)hip_stream;
  const dim3 grid(a.heads * blocks, batch);
  if (wide)
    ls::k_paged_fill<ls::u32x4><<<grid, 256, 0, st>>>(a, (const ls::u32x4*)from->k, (const ls::u32x4*)from->v, weights, (ls::u32x4*)pages->k, (ls::u32x4*)pages->v,
                                                  pages->weights, pages->places, pages->lens, pages->positions, blocks);
  else
    ls::k_paged_fill<uint32_t><<<grid, 256, 0, st>>>(a, (const uint32_t*)from->k, (const uint32_t*)from->v, weights, (uint32_t*)pages->k, (uint32_t*)pages->v,
                                                     pages->weights, pages->places, pages->lens, pages->positions, blocks);
  return launched(who);
}

size_t ls_paged_evict_scratch_bytes(const ls_heads* h, int layers, int batch, int keep, int max_len) {
  if (evict_error(h, layers, batch, keep, max_len)) return 0;
  const size_t units = evict_units(h, layers, batch), most = std::max(0, std::min(keep, max_len - keep));
  return (units * 4 + 15) / 16 * 16 + std::max((units * most * sizeof(int2) + 15) / 16 * 16, (size_t)16) + units * ls::key_groups(max_len) * 64 * 16 * 4;
}

ls_status ls_paged_evict(const ls_heads* h, int layers, const ls_pages* pages, int batch, int keep, int first, int recent, int max_len, void* scratch,
                         size_t scratch_bytes, void* hip_stream) {
  static const char* who = "ls_paged_evict";
  if (const char* e = evict_error(h, layers, batch, keep, max_len)) return bad(who, e);
  if (const char* e = ls::pages_error(h, pages, batch)) return bad(who, e);
  if (!pages->weights) return bad(who, "pages without weights and places");
  if (!pages->positions) return bad(who, "pages without positions, which lens do not give any more");
  if (first < 0 || recent < 0 || (int64_t)first + recent > keep) return bad(who, "first and recent are at least 0 and together at most keep");
  const uintptr_t at = (uintptr_t)pages->k | (uintptr_t)pages->v;
  if (at & 3) return bad(who, "a pool is not aligned to 4 bytes");
  if (!scratch || scratch_bytes < ls_paged_evict_scratch_bytes(h, layers, batch, keep, max_len)) {
    ls::set_last_error("%s: scratch is smaller than ls_paged_evict_scratch_bytes says", who);
    return LS_ERR_OOM;
  }
  if ((uintptr_t)scratch & 15) return bad(who, "scratch is not aligned to 16 bytes");
  if (max_len <= keep) return LS_OK;  // no sequence has more
  const size_t row = (size_t)h->head_dim * (h->dtype == LS_DTYPE_F32 ? 4 : 2), units = evict_units(h, layers, batch);
  const bool wide = row % 16 == 0 && (at & 15) == 0;
  const int pieces = (int)(row / (wide ? 16 : 4));
  ls::EvictArgs a;
  a.map = ls::map_of(pages);
  a.batch = batch; a.hkv = (int)h->n_kv_heads; a.layers = layers; a.keep = keep; a.first = first; a.recent = recent; a.max_len = max_len;
  a.most = std::min(keep, max_len - keep);
  a.weights = pages->weights; a.places = pages->places;
  a.count = (int32_t*)scratch;
  a.moves = (int2*)((char*)scratch + (units * 4 + 15) / 16 * 16);
  a.keys = (ls::u32x4*)((char*)a.moves + (units * a.most * sizeof(int2) + 15) / 16 * 16);
  a.groups = ls::key_groups(max_len);
  a.kc = pages->k; a.vc = pages->v; a.pieces = pieces; a.wide = wide;
  ls::launch_evict(a, units, pages->lens, (hipStream_t)hip_stream);
  return launched(who);
}

}  // extern "C"
