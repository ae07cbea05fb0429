// Attention of a tree of drafted tokens over a sequence's cache, with RoPE and the cache append.
//
// Node i of a sequence with c cached positions stands at position c + depth(i) and takes cache slot c + i.  Its query sees the c
// cached keys and the slots of the nodes on its path from the root, itself included.
//
// Here the kernels for every shape (the fast ones: tree_attn_mfma.hip): one rotates and appends the nodes' keys and values, one
// attends, a wavefront to a (row, query head), a lane to one or two pairs of dims, eight keys and values on their way at once.
// Bound by a wavefront's instructions, of which the sums over its lanes are half: 32 heads of 96 dims over 8, four sequences of 600
// keys, 12 nodes each 114 us in bf16, 110 in fp32 (a key at a time 253 and 335; sixteen at once no better).  The same of 128 dims
// takes 20 on the matrix cores.
#include "tree.hpp"

#include <algorithm>

namespace ls {

namespace {

template <class T>
__global__ void __launch_bounds__(256)
k_tree_append(const T* __restrict__ qkv, const float2* __restrict__ cs, const int32_t* __restrict__ cu, const int32_t* __restrict__ parents,
              const int32_t* __restrict__ seq_lens, int rows, int most, int hq, int hkv, int hd, int max_seq, T* __restrict__ kc, T* __restrict__ vc) {
  const int b = blockIdx.x, kh = blockIdx.y;
  TreeSeq t;
  if (!tree_seq(cu, seq_lens, b, rows, most, max_seq, t)) return;
  __shared__ int depth[TREE_MAX];
  const uint64_t path = tree_path(parents, t);
  if (threadIdx.x < 64) depth[threadIdx.x] = __builtin_popcountll(path) - 1;
  __syncthreads();
  const int half = hd >> 1;
  const size_t base = (((size_t)b * hkv + kh) * max_seq + t.ctx) * hd;
  for (int i = threadIdx.x; i < t.n * half; i += 256) {
    const int node = i / half, p = i - node * half;
    const T* row = qkv + (size_t)(t.row0 + node) * (hq + 2 * hkv) * hd;
    const T* k = row + (size_t)(hq + kh) * hd + 2 * p;
    const T* v = row + (size_t)(hq + hkv + kh) * hd + 2 * p;
    T* ko = kc + base + (size_t)node * hd + 2 * p;
    T* vo = vc + base + (size_t)node * hd + 2 * p;
    if (cs) {
      const float2 turn = cs[(size_t)(t.ctx + depth[node]) * half + p];
      const float u0 = to_f(k[0]), u1 = to_f(k[1]);
      ko[0] = from_f<T>(turn0(u0, u1, turn));
      ko[1] = from_f<T>(turn1(u0, u1, turn));
    } else {
      ko[0] = k[0];
      ko[1] = k[1];
    }
    vo[0] = v[0];
    vo[1] = v[1];
  }
}

// MAXP: pairs of a lane
template <class T, int MAXP>
__global__ void __launch_bounds__(64)
k_tree_attn(const T* __restrict__ qkv, const float2* __restrict__ cs, const int32_t* __restrict__ cu, const int32_t* __restrict__ parents,
            const int32_t* __restrict__ seq_lens, int rows, int most, int hq, int hkv, int hd, int max_seq, const T* __restrict__ kc,
            const T* __restrict__ vc, T* __restrict__ out) {
  typedef T T2 __attribute__((ext_vector_type(2), aligned(sizeof(T))));  // a row may start anywhere
  constexpr int AT_ONCE = 8;  // keys and values on their way
  const int b = blockIdx.x, node = blockIdx.y, h = blockIdx.z, lane = threadIdx.x, half = hd >> 1;
  TreeSeq t;
  const bool room = tree_seq(cu, seq_lens, b, rows, most, max_seq, t);
  if (node >= t.n) return;
  const int row0 = t.row0;
  T* o = out + (size_t)(row0 + node) * hq * hd + (size_t)h * hd;
  if (!room) {  // no room: the rows hold zeros
    for (int i = lane; i < hd; i += 64) o[i] = from_f<T>(0.f);
    return;
  }
  const uint64_t all = tree_path(parents, t);
  const uint64_t path = (uint64_t)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(all >> 32), node) << 32 |
                        (unsigned)__builtin_amdgcn_readlane((int)(unsigned)all, node);
  const int kh = h / (hq / hkv), pos = t.ctx + __builtin_popcountll(path) - 1;
  const T* q = qkv + (size_t)(row0 + node) * (hq + 2 * hkv) * hd + (size_t)h * hd;
  const float scale = 1.0f / sqrtf((float)hd);
  float q0[MAXP], q1[MAXP], a0[MAXP], a1[MAXP];
#pragma unroll
  for (int i = 0; i < MAXP; ++i) {
    const int p = lane + 64 * i;
    a0[i] = a1[i] = q0[i] = q1[i] = 0.f;
    if (p < half) {
      const float u0 = to_f(q[2 * p]), u1 = to_f(q[2 * p + 1]);
      const float2 turn = cs ? cs[(size_t)pos * half + p] : float2{1.f, 0.f};
      q0[i] = (cs ? turn0(u0, u1, turn) : u0) * scale;
      q1[i] = (cs ? turn1(u0, u1, turn) : u1) * scale;
    }
  }
  const T* kb = kc + ((size_t)b * hkv + kh) * max_seq * hd;
  const T* vb = vc + ((size_t)b * hkv + kh) * max_seq * hd;
  // Sums of AT_ONCE keys go into sums of NEAR times that, and those into the whole ones: one by one, equal weights next to a long sum are all
  // rounded the same way (60000 keys: off by 7e-4).
  constexpr int NEAR = 64;
  float m = -INFINITY, l = 0.f, far_l = 0.f, far0[MAXP] = {}, far1[MAXP] = {};
  for (int key0 = 0, turns = 1; key0 < t.ctx + t.n; key0 += AT_ONCE, ++turns) {
    T2 kr[AT_ONCE][MAXP], vr[AT_ONCE][MAXP];
    bool seen[AT_ONCE];
    float s[AT_ONCE], mn = m;
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      const int key = min(key0 + j, t.ctx + t.n - 1);
      seen[j] = key0 + j < t.ctx || (key0 + j < t.ctx + t.n && (path >> (key - t.ctx) & 1));
#pragma unroll
      for (int i = 0; i < MAXP; ++i) {
        const int p = min(lane + 64 * i, half - 1);
        const size_t at = (size_t)key * hd + 2 * p;
        kr[j][i] = *reinterpret_cast<const T2*>(kb + at);
        vr[j][i] = *reinterpret_cast<const T2*>(vb + at);
      }
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      s[j] = 0.f;
#pragma unroll
      for (int i = 0; i < MAXP; ++i)
        if (lane + 64 * i < half) s[j] = fmaf(q0[i], to_f(kr[j][i][0]), fmaf(q1[i], to_f(kr[j][i][1]), s[j]));
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) s[j] = wave_sum(s[j]);
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j)
      if (seen[j]) mn = fmaxf(mn, s[j]);
    const float corr = mn == -INFINITY ? 1.f : __expf(m - mn);
    float near_l = 0.f, near0[MAXP] = {}, near1[MAXP] = {};
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      if (!seen[j]) continue;
      const float w = s[j] == -INFINITY ? 0.f : __expf(s[j] - mn);
      near_l += w;
#pragma unroll
      for (int i = 0; i < MAXP; ++i) {
        near0[i] = fmaf(w, to_f(vr[j][i][0]), near0[i]);
        near1[i] = fmaf(w, to_f(vr[j][i][1]), near1[i]);
      }
    }
    l = fmaf(l, corr, near_l);
    far_l *= corr;
#pragma unroll
    for (int i = 0; i < MAXP; ++i) {
      a0[i] = fmaf(a0[i], corr, near0[i]);
      a1[i] = fmaf(a1[i], corr, near1[i]);
      far0[i] *= corr;
      far1[i] *= corr;
    }
    if (turns % NEAR == 0) {
      far_l += l;
      l = 0.f;
#pragma unroll
      for (int i = 0; i < MAXP; ++i) {
        far0[i] += a0[i];
        far1[i] += a1[i];
        a0[i] = a1[i] = 0.f;
      }
    }
    m = mn;
  }
#pragma unroll
  for (int i = 0; i < MAXP; ++i) {
    const int p = lane + 64 * i;
    if (p < half) {
      o[2 * p] = from_f<T>((far0[i] + a0[i]) / (far_l + l));
      o[2 * p + 1] = from_f<T>((far1[i] + a1[i]) / (far_l + l));
    }
  }
}

template <class T>
void launch_any(const TreeAttn& a, hipStream_t st) {
  k_tree_append<T><<<dim3(a.batch, a.hkv), 256, 0, st>>>((const T*)a.qkv, (const float2*)a.cs, a.cu, a.parents, a.seq_lens, a.rows, a.max_nodes, a.hq, a.hkv, a.hd,
                                                         a.max_seq, (T*)a.kc, (T*)a.vc);
  auto attn = a.hd <= 128 ? k_tree_attn<T, 1> : k_tree_attn<T, 2>;
  attn<<<dim3(a.batch, a.max_nodes, a.hq), 64, 0, st>>>((const T*)a.qkv, (const float2*)a.cs, a.cu, a.parents, a.seq_lens, a.rows, a.max_nodes, a.hq, a.hkv,
                                                        a.hd, a.max_seq, (const T*)a.kc, (const T*)a.vc, (T*)a.out);
}

// Chunks of a call.  One workgroup to a (sequence, kv head, block of columns) where they fill the chip.  Fewer with up to 32 columns are cut
// along the keys until each CU has one, in pieces of 128 keys at least: 7B, one sequence of 3000 keys, 26 nodes 18.3 us for 256
// workgroups, 20.0 for 512; 8 of 900 keys 33.3 and 35.9; 600 keys, 5 nodes in pieces of 128 10.3, of 256 11.4.  With more columns,
// whose wavefronts wait for each other, until all three places of a CU are taken, but not beyond: 70B, 16 ragged sequences of up to
// 3000 keys, 16 nodes 58 us for 768 workgroups, 59 for 512 and 58 for 1536; 13B, 16 of 1000 keys, 64 nodes (640 workgroups) 90, cut in
// two 110; 70B, one of 4000 keys, 64 nodes 33, in smaller pieces 39.  As more rows are joined their pieces have 256 keys: 70B, 4000 keys, 8 nodes 16.8, in pieces of 128 20.2.
TreeChunks chunks_for(const TreeAttn& a) {
  TreeChunks p;
  const int cols = a.max_nodes * (a.hq / a.hkv), wide = cols <= 16 ? 16 : cols <= 32 ? 32 : 64;
  const long base = (long)a.batch * a.hkv * ((cols + wide - 1) / wide);
  const long target = cols <= 32 ? 256 : 768, least = cols <= 32 ? 128 : 256;
  const long want = std::min(cols <= 32 ? (target + base - 1) / base : std::max(target / base, 1l), (a.max_keys + least - 1) / least);
  p.keys = (int)((a.max_keys + want - 1) / want + 63) / 64 * 64;
  p.n = (a.max_keys + p.keys - 1) / p.keys;
  return p;
}
size_t chunk_bytes(const TreeAttn& a, int n) { return (size_t)n * a.rows * a.hq * (a.hd + 2) * sizeof(float); }

bool fast(const TreeAttn& a) {
  const uintptr_t at = (uintptr_t)a.qkv | (uintptr_t)a.kc | (uintptr_t)a.vc | (uintptr_t)a.out | (uintptr_t)a.cs;
  return (a.hd == 64 || a.hd == 128) && (at & 15) == 0 && a.batch <= 65535 && (long)a.max_nodes * a.hq <= 65535;
}

}  // namespace

size_t tree_attn_scratch_bytes(const TreeAttn& a) {
  if (!fast(a)) return 0;
  const TreeChunks p = chunks_for(a);
  return p.n > 1 ? chunk_bytes(a, p.n) : 0;
}

void launch_tree_attn(uint32_t dt, const TreeAttn& a, hipStream_t st) {
  if (a.rows <= 0) return;
  if (fast(a)) {
    TreeChunks p = chunks_for(a);
    if (p.n > 1 && (!a.scratch || chunk_bytes(a, p.n) > a.scratch_bytes)) {  // as many as there is room for
      const int fit = a.scratch ? (int)(a.scratch_bytes / chunk_bytes(a, 1)) : 0;
      p.keys = ((a.max_keys + std::max(fit, 1) - 1) / std::max(fit, 1) + 63) / 64 * 64;
      p.n = (a.max_keys + p.keys - 1) / p.keys;
    }
    p.o = a.scratch;
    p.ml = a.scratch ? (float2*)(a.scratch + (size_t)p.n * a.rows * a.hq * a.hd) : nullptr;
    launch_tree_attn_mfma(dt, a, p, st);
    return;
  }
  if (dt == F32) launch_any<float>(a, st);
  else launch_any<bf16>(a, st);
}

}  // namespace ls
