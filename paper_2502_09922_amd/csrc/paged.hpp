// What the kernels of a cache in pages share.
#pragma once
#include "kernels.hpp"
#include "device_util.hpp"

namespace ls {

// Where the rows of sequences lie.
struct PageMap {
  const int32_t* lens = nullptr;
  const int32_t* positions = nullptr;  // or null: lens
  const int32_t* table = nullptr;
  int pages = 0, shift = 0, columns = 0;  // 1 << shift slots to a page
};

struct PagedAttn {
  PageMap map;
  const void* qkv = nullptr;
  const float* cs = nullptr;  // or null: rows come turned
  void *kc = nullptr, *vc = nullptr, *out = nullptr;
  float* weights = nullptr;
  int32_t* places = nullptr;
  int batch = 0, hq = 0, hkv = 0, hd = 0, size = 0, max_pos = 0, max_keys = 0;  // size: bytes of a value; max_keys: the new token's among them
  float* scratch = nullptr;
  size_t scratch_bytes = 0;
};
size_t paged_attn_scratch_bytes(const PagedAttn& a);
void launch_paged_attn(uint32_t dt, const PagedAttn& a, hipStream_t st);
void launch_paged_next(const PagedAttn& a, int32_t* lens, int32_t* positions, hipStream_t st);  // one more slot and position each

// Pieces of the contexts that workgroups of their own take, and where they leave their results: piece z of the row at `at` has place at + z * step.
// Dealt out beforehand (share == 0) a piece has `keys` slots of every sequence, at = row * hq + head, step = batch * hq.  Dealt out by the lengths
// (matrix cores), `share` workgroups get shares of about the same size and a place for 16 columns each: step = 16.
struct PagedPieces {
  static constexpr int SEQUENCES = 1024;  // at most, whose lengths a wavefront holds in registers to deal them out
  int n = 1, keys = 0;      // keys of a piece: a multiple of 64
  int share = 0;
  float* o = nullptr;       // [place][head_dim], not normalised
  float2* ml = nullptr;     // [place]: maximum in units of q k, sum
  int2* dealt = nullptr;    // [sequence]: first workgroup, pieces
  float* scores = nullptr;  // [row * hq + head][stride] q k of every slot, where weights are wanted
  int stride = 0;           // a multiple of 32
  int held = 0;             // from column to column of scores that stay in LDS
};
void launch_paged_attn_mfma(uint32_t dt, const PagedAttn& a, const PagedPieces& p, int most, hipStream_t st);  // head_dim 64 and 128, rows on 16 bytes

bool paged_joins_weights(const PagedAttn& a, const PagedPieces& p);  // by itself, without a join behind it

struct PagedSeq {
  int n, pos, page;  // slot and position of the new token, the slot's page
};

// Whether sequence b takes part.  `most`: slots that the call was made for (all of the table's where there are no weights).
__device__ __forceinline__ bool paged_seq(const PageMap& m, int b, int max_pos, bool turns, int most, PagedSeq& s) {
  s.n = m.lens[b];
  s.pos = m.positions ? m.positions[b] : s.n;
  s.page = -1;
  if (s.n < 0 || s.n >= most || s.n >> m.shift >= m.columns || s.pos < 0 || (turns && s.pos >= max_pos)) return false;
  s.page = m.table[(size_t)b * m.columns + (s.n >> m.shift)];
  return (unsigned)s.page < (unsigned)m.pages;
}

// First element of the rows of page `page` and kv head `kh`.
__device__ __forceinline__ size_t page_row0(int page, int hkv, int kh, int shift) { return ((size_t)page * hkv + kh) << shift; }

}  // namespace ls
