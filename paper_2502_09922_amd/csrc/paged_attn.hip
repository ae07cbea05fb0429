// Attention of one new token a sequence over a cache in pages, with RoPE and the append.
//
//   s_i = q k_i / sqrt(hd) over the slots 0..n, slot n the token's own;  o = sum_i softmax(s)_i v_i
//   weights[i] += sum over the query heads of a kv head of softmax(s)_i
//
// Here the kernel for every shape (the fast one: paged_attn_mfma.hip), which pieces a context is cut into, and the kernel that joins them
// and adds the weights up.  One wavefront to a (sequence, query head, piece), a lane to one or two pairs of dims, eight keys and values on
// their way at once; eight slots lie in one page, whose number is uniform.  Bound by a wavefront's instructions, as each query head reads the
// cache for itself: 96 dims, bf16, 40 heads over 40, 32 sequences of 1024 to 1087 slots 121 us (4.3 TB/s), 64 heads over 8, 64 of 128 to 2287 slots
// 697 (0.36 TB/s of what one reading takes).
#include "paged.hpp"

#include <algorithm>

namespace ls {

namespace {

// MAXP: pairs of a lane
template <class T, int MAXP>
__global__ void __launch_bounds__(64)
k_paged_attn(PageMap map, const T* __restrict__ qkv, const float2* __restrict__ cs, T* __restrict__ kc, T* __restrict__ vc, int32_t* __restrict__ places,
             T* __restrict__ out, int batch, int hq, int hkv, int hd, int max_pos, int most, PagedPieces p) {
  typedef T T2 __attribute__((ext_vector_type(2), aligned(sizeof(T))));  // a row may start anywhere
  constexpr int AT_ONCE = 8;  // keys and values on their way
  const int z = blockIdx.z, h = blockIdx.y, b = blockIdx.x, lane = threadIdx.x, half = hd >> 1;
  const int G = hq / hkv, kh = h / G;
  const size_t row = (size_t)b * hq + h;
  T* o = out + row * hd;
  PagedSeq t;
  if (!paged_seq(map, b, max_pos, cs != nullptr, most, t)) {
    if (z == 0)
      for (int i = lane; i < hd; i += 64) o[i] = from_f<T>(0.f);
    return;
  }
  const int lo = z * p.keys, keys = t.n + 1;
  if (lo >= keys) return;
  const int hi = z == p.n - 1 ? keys : min(lo + p.keys, keys);  // the last piece takes what is left
  const T* rows = qkv + (size_t)b * (hq + 2 * hkv) * hd;
  const bool own = hi == keys;  // the new token is among this piece's
  float q0[MAXP], q1[MAXP], k0[MAXP], k1[MAXP], v0[MAXP], v1[MAXP], a0[MAXP], a1[MAXP];
#pragma unroll
  for (int i = 0; i < MAXP; ++i) {
    const int at = lane + 64 * i;
    a0[i] = a1[i] = q0[i] = q1[i] = k0[i] = k1[i] = v0[i] = v1[i] = 0.f;
    if (at < half) {
      const float2 turn = cs ? cs[(size_t)t.pos * half + at] : float2{1.f, 0.f};
      auto turned = [&](const T* r, float& w0, float& w1) {
        const float u0 = to_f(r[2 * at]), u1 = to_f(r[2 * at + 1]);
        w0 = cs ? turn0(u0, u1, turn) : u0;
        w1 = cs ? turn1(u0, u1, turn) : u1;
      };
      turned(rows + (size_t)h * hd, q0[i], q1[i]);
      if (own) {
        turned(rows + (size_t)(hq + kh) * hd, k0[i], k1[i]);
        const T c0 = from_f<T>(k0[i]), c1 = from_f<T>(k1[i]);
        const T d0 = rows[(size_t)(hq + hkv + kh) * hd + 2 * at], d1 = rows[(size_t)(hq + hkv + kh) * hd + 2 * at + 1];
        k0[i] = to_f(c0);
        k1[i] = to_f(c1);
        v0[i] = to_f(d0);
        v1[i] = to_f(d1);
        if (h % G == 0) {
          const size_t to = (page_row0(t.page, hkv, kh, map.shift) + (t.n & ((1 << map.shift) - 1))) * hd + 2 * at;
          kc[to] = c0;
          kc[to + 1] = c1;
          vc[to] = d0;
          vc[to + 1] = d1;
        }
      }
    }
  }
  if (places && own && h % G == 0 && lane == 0) places[page_row0(t.page, hkv, kh, map.shift) + (t.n & ((1 << map.shift) - 1))] = t.pos;
  const float scale = 1.4426950408889634f / sqrtf((float)hd);  // q k -> exponent of 2
  const int32_t* entries = map.table + (size_t)b * map.columns;
  // Sums of AT_ONCE keys go into sums of NEAR times that, and those into the whole ones: one by one, equal weights next to a long sum
  // are all rounded the same way.
  constexpr int NEAR = 64;
  float m = -INFINITY, l = 0.f, far_l = 0.f, far0[MAXP] = {}, far1[MAXP] = {};
  for (int key0 = lo, turns = 1; key0 < hi; key0 += AT_ONCE, ++turns) {
    T2 kr[AT_ONCE][MAXP], vr[AT_ONCE][MAXP];
    const int page = entries[key0 >> map.shift];
    const bool there = (unsigned)page < (unsigned)map.pages;
    const size_t base = (page_row0(there ? page : 0, hkv, kh, map.shift) + (key0 & ((1 << map.shift) - 1))) * hd;
    bool seen[AT_ONCE];
    float s[AT_ONCE], mn = m;
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      seen[j] = there && key0 + j < hi;
#pragma unroll
      for (int i = 0; i < MAXP; ++i) {
        const size_t at = base + (size_t)j * hd + 2 * min(lane + 64 * i, half - 1);
        kr[j][i] = *reinterpret_cast<const T2*>(kc + at);
        vr[j][i] = *reinterpret_cast<const T2*>(vc + at);
      }
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      s[j] = 0.f;
      const bool new_one = own && key0 + j == t.n;
#pragma unroll
      for (int i = 0; i < MAXP; ++i)
        if (lane + 64 * i < half) s[j] = fmaf(q0[i], new_one ? k0[i] : to_f(kr[j][i][0]), fmaf(q1[i], new_one ? k1[i] : to_f(kr[j][i][1]), s[j]));
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) s[j] = wave_sum(s[j]);
    if (p.scores) {
      float mine = 0.f;
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) mine = lane == j ? s[j] : mine;
      if (lane < AT_ONCE && key0 + lane < hi) p.scores[row * p.stride + key0 + lane] = mine;
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j)
      if (seen[j]) mn = fmaxf(mn, s[j]);
    const float corr = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - mn) * scale);
    float near_l = 0.f, near0[MAXP] = {}, near1[MAXP] = {};
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
      if (!seen[j]) continue;
      const bool new_one = own && key0 + j == t.n;
      const float w = s[j] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((s[j] - mn) * scale);
      near_l += w;
#pragma unroll
      for (int i = 0; i < MAXP; ++i) {
        near0[i] = fmaf(w, new_one ? v0[i] : to_f(vr[j][i][0]), near0[i]);
        near1[i] = fmaf(w, new_one ? v1[i] : to_f(vr[j][i][1]), near1[i]);
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
  l += far_l;
  const bool whole = p.n == 1 || keys <= p.keys;
  const size_t at = (size_t)z * batch * hq + row;
  if ((!whole || p.scores) && lane == 0) p.ml[at] = float2{m, l};
#pragma unroll
  for (int i = 0; i < MAXP; ++i) {
    const int pair = lane + 64 * i;
    if (pair >= half) continue;
    const float n0 = far0[i] + a0[i], n1 = far1[i] + a1[i];
    if (whole) {
      o[2 * pair] = from_f<T>(n0 / l);
      o[2 * pair + 1] = from_f<T>(n1 / l);
    } else {
      p.o[at * hd + 2 * pair] = n0;
      p.o[at * hd + 2 * pair + 1] = n1;
    }
  }
}

// Sums over pieces: U of them at a time, NEAR times that, and those, so that equal ones next to a long sum are not all rounded the same way (4096 pieces,
// fp32: outputs off by 6.5e-5 of themselves, so 1e-6).
constexpr int NEAR = 16;

// Maximum and sum of a (sequence, query head) over its pieces, in their order, U of them on their way at once.
template <int U>
__device__ __forceinline__ float2 joined(const float2* __restrict__ ml, size_t step, int n, float scale) {
  float m = -INFINITY, den = 0.f, far = 0.f;
  for (int z0 = 0, turns = 1; z0 < n; z0 += U, ++turns) {
    float2 v[U];
    float top = m, sum = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = ml[min(z0 + u, n - 1) * step];
#pragma unroll
    for (int u = 0; u < U; ++u) top = fmaxf(top, v[u].x);
    const float corr = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - top) * scale);  // a sum without a maximum is 0, or no number
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (z0 + u < n) sum += v[u].y * (v[u].x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((v[u].x - top) * scale));
    den = fmaf(den, corr, sum);
    far *= corr;
    if (turns % NEAR == 0) {
      far += den;
      den = 0.f;
    }
    m = top;
  }
  return float2{m, far + den};
}

// The pieces' results, and the slots' weights.  Workgroups [0, out_blocks) of a sequence take its output, D dims to a thread, the others 256 slots
// of a kv head each, whose query heads' maxima and sums they join first.
template <class T, int D>
__global__ void __launch_bounds__(256)
k_paged_join(PageMap map, T* __restrict__ out, float* __restrict__ weights, int batch, int hq, int hkv, int hd, int max_pos, bool turns, int most, PagedPieces p,
             int out_blocks) {
  typedef T TD __attribute__((ext_vector_type(D), aligned(sizeof(T))));  // a row may start anywhere
  typedef float FD __attribute__((ext_vector_type(D)));
  constexpr int U = 8;  // pieces, or heads, on their way at once
  const int b = blockIdx.y, G = hq / hkv, blocks16 = (G + 15) / 16;
  const size_t step = p.share ? 16 : (size_t)batch * hq;
  const int2 dealt = p.share ? p.dealt[b] : int2{0, 0};
  auto place_of = [&](int h) {  // of a query head's first piece
    return p.share ? ((size_t)dealt.x + (size_t)(h / G * blocks16 + h % G / 16) * dealt.y) * 16 + h % G % 16 : (size_t)b * hq + h;
  };
  const float scale = 1.4426950408889634f / sqrtf((float)hd);
  PagedSeq t;
  if ((int)blockIdx.x < out_blocks) {
    const int i = min((int)(blockIdx.x * 256 + threadIdx.x), hq * hd / D - 1) * D, d = i % hd;
    const size_t row = (size_t)b * hq + i / hd, place = place_of(i / hd);
    float2 ml[U];
    FD v[U];
    auto load = [&](int z0) {  // the first of them before it is known how many there are
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const size_t at = place + min(z0 + u, (p.share ? dealt.y : p.n) - 1) * step;
        ml[u] = p.ml[at];
        v[u] = *reinterpret_cast<const FD*>(p.o + at * hd + d);
      }
    };
    load(0);
    if (!paged_seq(map, b, max_pos, turns, most, t)) return;
    const int n = p.share ? dealt.y : min((t.n + p.keys) / p.keys, p.n);
    if (n == 1) return;  // one piece writes the output itself
    float m = -INFINITY, den = 0.f, far_den = 0.f;
    FD num = 0.f, far_num = 0.f;
    for (int z0 = 0, times = 1; z0 < n; z0 += U, ++times) {
      if (z0) load(z0);
      float top = m, sum = 0.f;
      FD part = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) top = z0 + u < n ? fmaxf(top, ml[u].x) : top;
      const float corr = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - top) * scale);  // sums without a maximum are zeros, or no numbers
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (z0 + u < n) {
          const float wt = ml[u].x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((ml[u].x - top) * scale);
#pragma unroll
          for (int e = 0; e < D; ++e) part[e] += v[u][e] * wt;
          sum += ml[u].y * wt;
        }
      den = fmaf(den, corr, sum);
      far_den *= corr;
#pragma unroll
      for (int e = 0; e < D; ++e) num[e] = fmaf(num[e], corr, part[e]);
      far_num *= corr;
      if (times % NEAR == 0) {
        far_den += den;
        far_num += num;
        den = 0.f;
        num = 0.f;
      }
      m = top;
    }
    den += far_den;
    num += far_num;
    TD w;
#pragma unroll
    for (int e = 0; e < D; ++e) w[e] = from_f<T>(num[e] / den);
    *reinterpret_cast<TD*>(out + row * hd + d) = w;
    return;
  }
  const int blocks = (most + 255) / 256, item = blockIdx.x - out_blocks, kh = item / blocks, first = item % blocks * 256, slot = first + threadIdx.x;
  if (map.lens[b] < first) return;
  // pages and scores are asked for before it is known whether the sequence takes part
  const int page = map.table[(size_t)b * map.columns + min(slot >> map.shift, map.columns - 1)];
  float s[U];
  auto load = [&](int g0, int g) {
#pragma unroll
    for (int u = 0; u < U; ++u) s[u] = p.scores[((size_t)b * hq + kh * G + min(g0 + g + u, G - 1)) * p.stride + min(slot, p.stride - 1)];
  };
  load(0, 0);
  if (!paged_seq(map, b, max_pos, turns, most, t)) return;
  const int keys = t.n + 1, n = p.share ? dealt.y : min((t.n + p.keys) / p.keys, p.n);
  const bool there = slot < keys && (unsigned)page < (unsigned)map.pages;
  const size_t at = page_row0(there ? page : 0, hkv, kh, map.shift) + (slot & ((1 << map.shift) - 1));
  const float had = there && slot != t.n ? weights[at] : 0.f;
  __shared__ float2 heads[64];  // maximum, 1 / sum
  float got = 0.f;
  for (int g0 = 0; g0 < G; g0 += 64) {
    const int count = min(64, G - g0);
    if (g0) load(g0, 0);
    if (g0) __syncthreads();
    if ((int)threadIdx.x < count) {
      const float2 all = joined<U>(p.ml + place_of(kh * G + g0 + threadIdx.x), step, n, scale);
      heads[threadIdx.x] = float2{all.x == -INFINITY ? 0.f : all.x, 1.f / all.y};
    }
    __syncthreads();
    for (int g = 0; g < count; g += U) {
      if (g) load(g0, g);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (g + u < count) got += __builtin_amdgcn_exp2f((s[u] - heads[g + u].x) * scale) * heads[g + u].y;
    }
  }
  if (there) weights[at] = had + got;
}

template <class T>
void launch_any(const PagedAttn& a, const PagedPieces& p, int most, hipStream_t st) {
  auto attn = a.hd <= 128 ? k_paged_attn<T, 1> : k_paged_attn<T, 2>;
  attn<<<dim3(a.batch, a.hq, p.n), 64, 0, st>>>(a.map, (const T*)a.qkv, (const float2*)a.cs, (T*)a.kc, (T*)a.vc, a.places, (T*)a.out, a.batch, a.hq, a.hkv, a.hd,
                                                a.max_pos, most, p);
}

bool fast(const PagedAttn& a) {
  const uintptr_t at = (uintptr_t)a.qkv | (uintptr_t)a.kc | (uintptr_t)a.vc | (uintptr_t)a.out | (uintptr_t)a.cs;
  return (a.hd == 64 || a.hd == 128) && (at & 15) == 0 && a.hq <= 65535;
}

size_t up16(size_t n) { return (n + 15) / 16 * 16; }
int score_stride(const PagedAttn& a) { return (a.max_keys + 31) / 32 * 32; }
size_t score_bytes(const PagedAttn& a) { return a.weights ? (size_t)a.batch * a.hq * score_stride(a) * sizeof(float) : 0; }
size_t place_bytes(const PagedAttn& a) { return (size_t)(a.hd + 2) * sizeof(float); }
// Of partial results, and of what is beside them.
size_t piece_bytes(const PagedAttn& a, const PagedPieces& p) {
  return p.share ? p.share * 16 * place_bytes(a) + up16(a.batch * sizeof(int2)) : (size_t)p.n * a.batch * a.hq * place_bytes(a);
}

// Pieces of a call's contexts, as far as `room` bytes go.  On the matrix cores:
//   - Where a kv head's keys and values of a sequence are at most ONE bytes, one workgroup each and no second launch: 8 kv heads, bf16, 128 dims,
//     600 slots 10.2 us, in pieces of 128 slots 11.7 (900 slots 12.1 and 11.7); 64 dims, 1200 slots 11.2 and 11.4; fp32, 128 dims, 300 slots 11.5
//     and 11.8, 400 slots 13.7 and 11.8.
//   - Where some may be longer than LONG bytes, workgroups get shares by the lengths that the device knows: of 32 sequences of 500 slots and one of 16000, 64
//     heads over 8, the long one's 8 workgroups take 191 us, shared out 39; 64 of 300 and two of 3500 51 and 31.  It costs a microsecond in
//     front and the second launch: 64 of 5000 slots 200 us uncut, 209 shared out; 64 of 2287 93 and 103.
//   - Otherwise in equal pieces until a CU each has one: 7B, one sequence of 3000 slots 14.9 us, 16.6 with two to a CU.  Where lengths differ the longest
//     one's pieces are what the launch waits for: 32 heads, fp32, 700, 596, 240 and 632 slots 24 tiles, of which an even share were 17.
PagedPieces pieces_for(const PagedAttn& a, size_t room) {
  PagedPieces p;
  p.keys = (a.max_keys + 63) / 64 * 64;
  const long units = (long)a.hkv * ((a.hq / a.hkv + 15) / 16), base = a.batch * units;
  if (fast(a)) {
    constexpr long CUS = 256, ONE = 300 << 10, LONG = 1500 << 10;
    const long bytes = (long)a.max_keys * a.hd * 2 * a.size;
    if (bytes <= ONE) return p;
    if (a.batch > 1 && bytes > LONG && a.batch <= PagedPieces::SEQUENCES && base <= (1 << 16)) {
      p.share = (int)(2 * base <= CUS ? CUS : base <= CUS ? 2 * CUS : base + 2 * CUS);
      const size_t each = 16 * place_bytes(a), beside = up16(a.batch * sizeof(int2));
      if (piece_bytes(a, p) > room) p.share = room > beside ? (int)((room - beside) / each) : 0;
      if (p.share > base) return p;
      p.share = 0;
    }
    const long fit = (long)std::min(room / ((size_t)a.batch * a.hq * place_bytes(a)), (size_t)1 << 20);
    const long want = std::min({std::max(CUS / base, 1l), (a.max_keys + 127l) / 128, std::max(fit, 1l)});
    p.keys = (int)((a.max_keys + want - 1) / want + 63) / 64 * 64;
    p.n = (a.max_keys + p.keys - 1) / p.keys;
    return p;
  }
  const long rows = (long)a.batch * a.hq, fit = (long)std::min(room / (rows * place_bytes(a)), (size_t)1 << 20);
  const long want = std::min({std::max(4096 / rows, 1l), (a.max_keys + 127l) / 128, std::max(fit, 1l)});
  p.keys = (int)((a.max_keys + want - 1) / want + 63) / 64 * 64;
  p.n = (a.max_keys + p.keys - 1) / p.keys;
  return p;
}

}  // namespace

size_t paged_attn_scratch_bytes(const PagedAttn& a) {
  const PagedPieces p = pieces_for(a, SIZE_MAX);
  // with weights, room for one piece of the kernel for every shape, which buffers that are not known here may want
  const size_t least = a.weights ? (size_t)a.batch * a.hq * place_bytes(a) : 0;
  return score_bytes(a) + std::max(p.n > 1 || p.share ? piece_bytes(a, p) : 0, least);
}

void launch_paged_attn(uint32_t dt, const PagedAttn& a, hipStream_t st) {
  const int most = a.weights ? a.max_keys : INT32_MAX;
  PagedPieces p = pieces_for(a, a.scratch ? a.scratch_bytes - score_bytes(a) : 0);
  if (a.scratch) {
    float* at = a.scratch;
    if (a.weights) {
      p.scores = at;
      p.stride = score_stride(a);
      at += (size_t)a.batch * a.hq * p.stride;
    }
    if (p.share) {
      p.dealt = (int2*)at;
      at += up16(a.batch * sizeof(int2)) / sizeof(float);
    }
    p.o = at;
    p.ml = (float2*)(at + (p.share ? (size_t)p.share * 16 : (size_t)p.n * a.batch * a.hq) * a.hd);
  }
  if (fast(a)) launch_paged_attn_mfma(dt, a, p, most, st);
  else if (dt == F32) launch_any<float>(a, p, most, st);
  else launch_any<bf16>(a, p, most, st);
  const bool cut = p.n > 1 || p.share;
  if (!cut && (!a.weights || (fast(a) && paged_joins_weights(a, p)))) return;
  const int D = a.hd % 4 ? 2 : 4, out_blocks = cut ? (a.hq * a.hd / D + 255) / 256 : 0, slots = a.weights ? a.hkv * ((a.max_keys + 255) / 256) : 0;
  const dim3 grid(out_blocks + slots, a.batch);
  auto join = [&](auto* kernel, auto* out) {
    kernel<<<grid, 256, 0, st>>>(a.map, out, a.weights, a.batch, a.hq, a.hkv, a.hd, a.max_pos, a.cs != nullptr, most, p, out_blocks);
  };
  if (dt == F32) join(D == 4 ? k_paged_join<float, 4> : k_paged_join<float, 2>, (float*)a.out);
  else join(D == 4 ? k_paged_join<bf16, 4> : k_paged_join<bf16, 2>, (bf16*)a.out);
}

namespace {

__global__ void __launch_bounds__(256)
k_paged_next(PageMap map, int32_t* lens, int32_t* positions, int batch, int max_pos, int most) {
  const int b = blockIdx.x * 256 + threadIdx.x;
  PagedSeq t;
  if (b >= batch || !paged_seq(map, b, max_pos, true, most, t)) return;
  lens[b] = t.n + 1;
  if (positions) positions[b] = t.pos + 1;
}

}  // namespace

void launch_paged_next(const PagedAttn& a, int32_t* lens, int32_t* positions, hipStream_t st) {
  k_paged_next<<<(a.batch + 255) / 256, 256, 0, st>>>(a.map, lens, positions, a.batch, a.max_pos, a.weights ? a.max_keys : INT32_MAX);
}

}  // namespace ls
