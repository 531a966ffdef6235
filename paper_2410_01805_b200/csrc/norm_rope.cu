// Norms of queries and keys for each head, rotation, cache append; and the gradients.  Bound by memory: every element is read
// and written once.
#include <type_traits>

#include "../../include/locret.h"
#include "common.cuh"
#include "paged.cuh"

namespace locret {
namespace {

struct NormRope {
  const void *q, *k, *v, *g_q, *g_k;
  void *q_out, *k_out;
  long long q_token, k_token, v_token, q_out_token, k_out_token;
  int q_head, k_head, v_head, q_out_head, k_out_head;   // (32 bits: one instruction less per row and product)
  const int32_t *positions;
  const uint64_t *turns;
  const int64_t *slots;
  int32_t *status;
  PageView pages;
  int n_tok, h, h_kv, d, rot;
  float factor, eps, inv_d;
};

// Cosine and sine of position * turns / 2^64 turns.  The product's low 64 bits are the exact fraction of a turn at every
// position; its upper 32 bits, taken as the nearest quarter turn and a rest of at most an eighth, are the angle to 2^-32 turns.
// On |x| <= pi / 4 the Taylor polynomials of degree 9 and 10 are off by 2e-9 and 1e-10.
__device__ __forceinline__ float2 cos_sin(uint64_t turns, int position, float factor) {
  const uint32_t top = (uint32_t)((turns * (uint64_t)(int64_t)position) >> 32);
  const uint32_t quarter = (top + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(top - (quarter << 30)) * 1.4629180792671596e-9f;   // 2 pi / 2^32
  const float x2 = x * x;
  float s = fmaf(x2, 1.0f / 362880, -1.0f / 5040), c = fmaf(x2, -1.0f / 3628800, 1.0f / 40320);
  s = fmaf(x2, s, 1.0f / 120);
  c = fmaf(x2, c, -1.0f / 720);
  s = fmaf(x2, s, -1.0f / 6);
  c = fmaf(x2, c, 1.0f / 24);
  s = fmaf(x2 * x, s, x);
  c = fmaf(x2, c, -0.5f);
  c = fmaf(x2, c, 1.0f);
  const float cc = quarter & 1 ? s : c, ss = quarter & 1 ? c : s;
  return make_float2((quarter + 1) & 2 ? -cc * factor : cc * factor, quarter & 2 ? -ss * factor : ss * factor);
}

// A row (one head of one token) is d / E items of E elements, one for each lane of a group.  Item j < rot / E holds E / 2 pairs
// whole - with half rotation, E / 2 elements of either half - so a rotation needs no other lane; two accesses an item, of 16
// bytes (E = 16) or 8, neighbouring lanes next to each other.
// E = 16 where d and rot are multiples of 16, 8 otherwise: what bounds the kernels beside memory is the number of
// instructions, and a row's addresses, sums over lanes and conversions cost the same for half the elements (in one block per few
// tokens with the rotation in shared memory, 8191 tokens of the Llama shape took 58.7 us with E = 8 and 43.4 with 16, the gradients
// of 10240 tokens 137 and 91).
template <int E>
struct Item {
  int a, b;       // offsets of its two runs of E / 2 elements
  bool rotates, there;
  template <int I>
  static __device__ __forceinline__ Item of(int j, int d, int rot) {
    Item it;
    it.there = j * E < d;
    it.rotates = j * E < rot;
    it.a = it.rotates && !I ? E / 2 * j : E * j;
    it.b = it.rotates && !I ? rot / 2 + E / 2 * j : E * j + E / 2;
    return it;
  }
};

// E 16-bit numbers as they are loaded and stored: two vectors
template <int E> struct Raw;
template <> struct Raw<8> { uint2 v[2]; };
template <> struct Raw<16> { uint4 v[2]; };

template <typename T, int E>
__device__ __forceinline__ Raw<E> load_item(const T *row, const Item<E> &it, bool ok) {
  typedef decltype(Raw<E>::v[0]) Ref;
  typedef typename std::remove_reference<Ref>::type V;
  Raw<E> r = {};
  if (ok && it.there) {
    r.v[0] = *reinterpret_cast<const V *>(row + it.a);
    r.v[1] = *reinterpret_cast<const V *>(row + it.b);
  }
  return r;
}
template <typename T, int E>
__device__ __forceinline__ void store_item(T *a, int ab, const Raw<E> &r) {   // (as Ring::request)
  typedef typename std::remove_cv<typename std::remove_reference<decltype(r.v[0])>::type>::type V;
  *reinterpret_cast<V *>(a) = r.v[0];
  *reinterpret_cast<V *>(a + ab) = r.v[1];
}
// A lane's ring of stages in shared memory, N items each, filled by asynchronous copies: what a warp has on its way costs no
// registers, and every lane reads what it copied itself, so nothing else is waited for.
template <int E, int N, int STAGES>
struct Ring {
  typedef typename std::remove_reference<decltype(Raw<E>::v[0])>::type V;
  V v[STAGES][N][2][32];
  // a: the item's first run; ab: how far behind it the second lies
  template <typename T>
  __device__ __forceinline__ void request(int stage, int n, const T *a, int ab, bool ok, const T *safe) {
    const int lane = threadIdx.x & 31, bytes = ok ? (int)sizeof(V) : 0;   // (0: nothing is read, the place is filled with zeros)
    const T *from = ok ? a : safe;
    copy(&v[stage][n][0][lane], from, bytes);
    copy(&v[stage][n][1][lane], from + ab, bytes);
  }
  __device__ __forceinline__ Raw<E> get(int stage, int n) const {
    const int lane = threadIdx.x & 31;
    Raw<E> r;
    r.v[0] = v[stage][n][0][lane];
    r.v[1] = v[stage][n][1][lane];
    return r;
  }
  static __device__ __forceinline__ void copy(V *to, const void *from, int bytes) {
    if (E == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(smem_u32(to)), "l"(from), "r"(bytes));
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;\n" ::"r"(smem_u32(to)), "l"(from), "r"(bytes));
  }
};

// The items' arithmetic goes two elements at a time (packed fp32): what bounds the kernels beside memory is the number of
// instructions.  P2[i] holds x[2i] and x[2i+1].
template <int E> struct P2 { uint64_t v[E / 2]; };
__device__ __forceinline__ uint64_t mul_f32x2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t both(float x) { return pack_f32x2(x, x); }
__device__ __forceinline__ uint64_t swapped(uint64_t a) {
  float lo, hi;
  unpack_f32x2(a, lo, hi);
  return pack_f32x2(hi, lo);
}
template <typename T, int E>
__device__ __forceinline__ P2<E> unpack2(const Raw<E> &r) {
  const uint32_t *w = reinterpret_cast<const uint32_t *>(&r);
  P2<E> x;
#pragma unroll
  for (int i = 0; i < E / 2; i++) {
    const float2 f = Half2<T>::unpack(w[i]);
    x.v[i] = pack_f32x2(f.x, f.y);
  }
  return x;
}
template <typename T, int E>
__device__ __forceinline__ Raw<E> pack2(const P2<E> &x) {
  Raw<E> r;
  uint32_t *w = reinterpret_cast<uint32_t *>(&r);
#pragma unroll
  for (int i = 0; i < E / 2; i++) {
    float lo, hi;
    unpack_f32x2(x.v[i], lo, hi);
    w[i] = Half2<T>::pack(lo, hi);
  }
  return r;
}
template <int E>
__device__ __forceinline__ float dot2(const P2<E> &a, const P2<E> &b) {
  uint64_t s = mul_f32x2(a.v[0], b.v[0]);
#pragma unroll
  for (int i = 1; i < E / 2; i++) s = fma_f32x2(a.v[i], b.v[i], s);
  float lo, hi;
  unpack_f32x2(s, lo, hi);
  return lo + hi;
}

// A lane's pairs of one token as factors: out = x * same + partner(x) * other, where the partner of an element is the other one
// of its pair.  With the gains g in them (forward): same = g c, other = -+ g(partner) s; back (gradients): same = c, other = +- s.
template <int E> struct Turn { P2<E> same, other; };
template <int E, int I>
__device__ __forceinline__ P2<E> turned(const P2<E> &x, const Turn<E> &t) {
  P2<E> y;
#pragma unroll
  for (int i = 0; i < E / 2; i++) {
    const uint64_t partner = I ? swapped(x.v[i]) : x.v[(i + E / 4) % (E / 2)];
    y.v[i] = fma_f32x2(partner, t.other.v[i], mul_f32x2(x.v[i], t.same.v[i]));
  }
  return y;
}
// pairs: the token's; gain: of the lane's elements (ones where there is none)
template <int E, int I, bool BACK>
__device__ __forceinline__ Turn<E> turn_of(const float2 *pairs, const Item<E> &it, int j, const P2<E> &gain) {
  Turn<E> t;
#pragma unroll
  for (int i = 0; i < E / 2; i += 2) {
    const float4 cs = it.rotates ? *reinterpret_cast<const float4 *>(pairs + E / 2 * j + i) : make_float4(1.f, 0.f, 1.f, 0.f);
    const float s0 = BACK ? -cs.y : cs.y, s1 = BACK ? -cs.w : cs.w;
    if (I) {   // pairs i, i + 1: elements 2i, 2i + 1 and the two behind them
      t.same.v[i] = mul_f32x2(gain.v[i], both(cs.x));
      t.same.v[i + 1] = mul_f32x2(gain.v[i + 1], both(cs.z));
      t.other.v[i] = mul_f32x2(swapped(gain.v[i]), pack_f32x2(-s0, s0));
      t.other.v[i + 1] = mul_f32x2(swapped(gain.v[i + 1]), pack_f32x2(-s1, s1));
    } else {   // elements i, i + 1 and the same behind half of them
      const uint64_t c2 = pack_f32x2(cs.x, cs.z);
      t.same.v[i / 2] = mul_f32x2(gain.v[i / 2], c2);
      t.same.v[i / 2 + E / 4] = mul_f32x2(gain.v[i / 2 + E / 4], c2);
      t.other.v[i / 2] = mul_f32x2(gain.v[i / 2 + E / 4], pack_f32x2(-s0, -s1));
      t.other.v[i / 2 + E / 4] = mul_f32x2(gain.v[i / 2], pack_f32x2(s0, s1));
    }
  }
  return t;
}
template <int E>
__device__ __forceinline__ P2<E> ones() {
  P2<E> x;
#pragma unroll
  for (int i = 0; i < E / 2; i++) x.v[i] = both(1.f);
  return x;
}

template <int G>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The warp's cosines and sines of a token at `position`, into its part of shared memory.
__device__ __forceinline__ void fill_pairs(float2 *s, const NormRope &p, int position) {
  __syncwarp();
  for (int i = threadIdx.x & 31; i < p.rot / 2; i += 32) s[i] = cos_sin(p.turns[i], position, p.factor);
  __syncwarp();
}

// A warp takes rows of one token, 32 / G at a time (G lanes a row, the power of two that covers d / E): a step is that many
// heads of queries, keys or (with pages) values, and a token's steps are divided over `slices` warps.  What the token's
// rotation and the gains make of a lane's elements stays in registers; nothing but the warp itself is waited for.  8191 tokens of
// the Llama shape with norms and append: 37.8 us for 201 MB, 5.3 TB/s, 0.81 of the copy rate; what is left is instructions (230 a
// step of four rows) and the last wave of blocks.  A persistent grid with rings across tokens: 36.8, but 200 tokens 5.3 -> 6.7.
constexpr int NR_THREADS = 128, NR_WARPS = NR_THREADS / 32;

constexpr int NR_STAGES = 4;   // steps a warp has on their way, and the one it works on (39.0 us; six 41.0, nine 44.8)

template <typename T, int E, int G, int I>
__global__ void __launch_bounds__(NR_THREADS, 5)
norm_rope_kernel(const __grid_constant__ NormRope p, int slices) {
  constexpr int R = 32 / G;
  __shared__ __align__(16) float2 pairs[NR_WARPS][128];
  __shared__ Ring<E, 1, NR_STAGES> rings[NR_WARPS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane % G, row = lane / G;
  const long long unit = (long long)blockIdx.x * NR_WARPS + warp, tok = unit / slices;
  if (tok >= p.n_tok) return;
  const int slice = (int)(unit - tok * slices);
  const int q_steps = (p.h + R - 1) / R, k_steps = (p.h_kv + R - 1) / R, steps = q_steps + (p.pages.k ? 2 : 1) * k_steps;
  const int s0 = (int)((long long)steps * slice / slices), s1 = (int)((long long)steps * (slice + 1) / slices);
  const Item<E> it = Item<E>::template of<I>(j, p.d, p.rot);
  const int ab = it.b - it.a;
  Ring<E, 1, NR_STAGES> &ring = rings[warp];
  const T *const safe = static_cast<const T *>(p.q);
  // what is requested: the lane's item in row `head` of one kind, R heads further with every step
  int ask_left = s1 - s0, ask_kind, ask_head, ask_rows, fill = 0;
  const T *ask_at;
  long long ask_by;
  auto ask_from = [&](int kind, int step) {
    ask_kind = kind;
    ask_head = step * R + row;
    ask_rows = kind == 0 ? p.h : p.h_kv;
    const int stride = kind == 0 ? p.q_head : kind == 1 ? p.k_head : p.v_head;
    ask_at = static_cast<const T *>(kind == 0 ? p.q : kind == 1 ? p.k : p.v) +
             tok * (kind == 0 ? p.q_token : kind == 1 ? p.k_token : p.v_token) + (long long)ask_head * stride + it.a;
    ask_by = (long long)R * stride;
  };
  auto ask = [&]() {
    if (ask_left > 0) {
      ring.request(fill, 0, ask_at, ab, ask_head < ask_rows && it.there, safe);
      ask_at += ask_by;
      ask_head += R;
      if (--ask_left > 0 && ask_head - row >= ask_rows) ask_from(ask_kind + 1, 0);
    }
    cp_async_commit();
    fill = fill + 1 == NR_STAGES ? 0 : fill + 1;
  };
  const int kind0 = s0 < q_steps ? 0 : s0 < q_steps + k_steps ? 1 : 2;
  const int step0 = s0 - (kind0 == 0 ? 0 : kind0 == 1 ? q_steps : q_steps + k_steps);
  ask_from(kind0, step0);
#pragma unroll
  for (int i = 0; i < NR_STAGES - 1; i++) ask();
  // the token's place in the pool
  long long place = -1;
  if (p.pages.k) {
    const int64_t slot = p.slots[tok];
    if (slot >= 0) {
      const int64_t page = slot <= INT32_MAX ? (int64_t)p.pages.by_size.div((int)slot) : slot / p.pages.page_size;
      if (page < p.pages.n_pages) place = page * p.pages.page_stride + (slot - page * p.pages.page_size) * p.pages.token_stride;
      else if (lane == 0) report(p.status, LOCRET_ERR_INVALID);
    }
  }
  fill_pairs(pairs[warp], p, p.rot ? p.positions[tok] : 0);

  int left = s1 - s0, kind = kind0, step = step0, stage = 0;
  while (left > 0) {   // (a kind)
    const int rows = kind == 0 ? p.h : p.h_kv, n = min(left, (rows + R - 1) / R - step);
    left -= n;
    int head = step * R + row;
    const T *const g = static_cast<const T *>(kind == 0 ? p.g_q : kind == 1 ? p.g_k : nullptr);
    const int dst_stride = kind == 0 ? p.q_out_head : p.k_out_head;
    T *dst = static_cast<T *>(kind == 0 ? p.q_out : kind == 1 ? p.k_out : nullptr);
    if (dst) dst += tok * (kind == 0 ? p.q_out_token : p.k_out_token) + (long long)head * dst_stride + it.a;
    T *pool = kind && place >= 0 ? static_cast<T *>(kind == 1 ? p.pages.k : p.pages.v) : nullptr;
    if (pool) pool += place + head * p.pages.head_stride + it.a;
    Turn<E> turn;
    if (kind < 2) turn = turn_of<E, I, false>(pairs[warp], it, j, g ? unpack2<T>(load_item(g, it, true)) : ones<E>());
    for (int i = 0; i < n; i++) {
      cp_async_wait<NR_STAGES - 2>();
      Raw<E> out = ring.get(stage, 0);
      stage = stage + 1 == NR_STAGES ? 0 : stage + 1;
      ask();   // (into the stage that the last step was done with)
      if (kind < 2) {
        P2<E> x = unpack2<T>(out);
        if (g) {
          const float ss = group_sum<G>(dot2(x, x));
          const uint64_t rstd = both(rsqrtf(fmaf(ss, p.inv_d, p.eps)));
#pragma unroll
          for (int e = 0; e < E / 2; e++) x.v[e] = mul_f32x2(x.v[e], rstd);
        }
        if (it.rotates) {
          x = turned<E, I>(x, turn);
        } else {
#pragma unroll
          for (int e = 0; e < E / 2; e++) x.v[e] = mul_f32x2(x.v[e], turn.same.v[e]);
        }
        out = pack2<T>(x);
      }
      const bool ok = head < rows && it.there;
      head += R;
      if (dst) {
        if (ok) store_item(dst, ab, out);
        dst += (long long)R * dst_stride;
      }
      if (pool) {
        if (ok) store_item(pool, ab, out);
        pool += R * p.pages.head_stride;
      }
    }
    kind++;
    step = 0;
  }
}

// ---------------------------------------------------------------- gradients
//   t = R^T dy,  n = x rstd,  d_g = sum t n,  dx = rstd (t g - n mean(t g n));   without a norm dx = t
// A persistent grid whose blocks are dealt to queries and keys by their rows; a warp takes the rows of one token after the
// other, adds up t n in registers, and every block writes one partial sum; a second kernel adds those, in the order of the blocks.
// 10240 tokens of the Llama shape: 62.4 us for 315 MB, 5.0 TB/s, 0.77 of the copy rate, bound by instructions at twelve warps an SM
// (150 registers: rotation, gains and their sums); two stages of a ring or four make no difference.
constexpr int NRG_THREADS = 128, NRG_WARPS = NRG_THREADS / 32, NRG_STAGES = 4;
struct Part { int blocks, slices; };   // of one kind: its blocks, and warps that divide a token's rows

template <typename T, int E, int G, int I>
__global__ void __launch_bounds__(NRG_THREADS, E == 16 ? 3 : 4)
norm_rope_grad_kernel(const __grid_constant__ NormRope p, const __grid_constant__ Part q_part, const __grid_constant__ Part k_part,
                      T *d_q, T *d_k, float *partial) {
  constexpr int R = 32 / G, GROUPS = NRG_WARPS * R;
  __shared__ __align__(16) float2 pairs[NRG_WARPS][128];
  __shared__ Ring<E, 2, NRG_STAGES> rings[NRG_WARPS];
  __shared__ float sums[GROUPS][G * E];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, j = lane % G, row = lane / G;
  const int kind = blockIdx.x < q_part.blocks ? 0 : 1;
  const Part part = kind == 0 ? q_part : k_part;
  const int b = blockIdx.x - (kind == 0 ? 0 : q_part.blocks), rows = kind == 0 ? p.h : p.h_kv;
  const T *dy = static_cast<const T *>(kind == 0 ? p.q_out : p.k_out), *src = static_cast<const T *>(kind == 0 ? p.q : p.k);
  const long long dy_token = kind == 0 ? p.q_out_token : p.k_out_token, src_token = kind == 0 ? p.q_token : p.k_token;
  const int dy_head = kind == 0 ? p.q_out_head : p.k_out_head, src_head = kind == 0 ? p.q_head : p.k_head;
  T *dx = kind == 0 ? d_q : d_k;
  const T *g = static_cast<const T *>(kind == 0 ? p.g_q : p.g_k);
  const Item<E> it = Item<E>::template of<I>(j, p.d, p.rot);
  const Raw<E> gain_raw = load_item(g, it, g != nullptr);
  P2<E> dg = {};
  pdl_launch_dependents();
  const int steps = (rows + R - 1) / R;
  const long long units = (long long)p.n_tok * part.slices, stride = (long long)part.blocks * NRG_WARPS;
  Ring<E, 2, NRG_STAGES> &ring = rings[warp];
  const int ab = it.b - it.a;
  auto steps_of = [&](long long unit, long long &tok, int &s0, int &s1) {
    tok = unit;
    s0 = 0;
    s1 = steps;
    if (part.slices > 1) {   // (few tokens)
      tok = unit / part.slices;
      const int slice = (int)(unit - tok * part.slices);
      s0 = (int)((long long)steps * slice / part.slices);
      s1 = (int)((long long)steps * (slice + 1) / part.slices);
    }
  };
  // what is requested next: it runs ahead over the warp's tokens
  long long ask_unit = (long long)b * NRG_WARPS + warp;
  int ask_left = 0, ask_head = 0, fill = 0;
  const T *ask_dy = dy, *ask_x = src;
  const long long dy_by = (long long)R * dy_head, x_by = (long long)R * src_head;
  auto ask_from = [&]() {
    if (ask_unit >= units) return;
    long long tok;
    int s0, s1;
    steps_of(ask_unit, tok, s0, s1);
    ask_left = s1 - s0;
    ask_head = s0 * R + row;
    ask_dy = dy + tok * dy_token + (long long)ask_head * dy_head + it.a;
    ask_x = src + tok * src_token + (long long)ask_head * src_head + it.a;
  };
  ask_from();
  auto ask = [&]() {
    if (ask_left > 0) {
      const bool ok = ask_head < rows && it.there;
      ring.request(fill, 0, ask_dy, ab, ok, dy);
      if (g) ring.request(fill, 1, ask_x, ab, ok, src);
      ask_dy += dy_by;
      ask_x += x_by;
      ask_head += R;
      if (--ask_left == 0) {
        ask_unit += stride;
        ask_from();
      }
    }
    cp_async_commit();
    fill = fill + 1 == NRG_STAGES ? 0 : fill + 1;
  };
#pragma unroll
  for (int i = 0; i < NRG_STAGES - 1; i++) ask();
  int stage = 0;
  long long unit = (long long)b * NRG_WARPS + warp;
  auto position_of = [&](long long unit) { return unit < units && p.rot ? p.positions[part.slices > 1 ? unit / part.slices : unit] : 0; };
  int next_position = position_of(unit);
  for (; unit < units; unit += stride) {
    long long tok;
    int s0, s1;
    steps_of(unit, tok, s0, s1);
    const int position = next_position;
    next_position = position_of(unit + stride);
    fill_pairs(pairs[warp], p, position);
    const Turn<E> turn = turn_of<E, I, true>(pairs[warp], it, j, ones<E>());
    int head = s0 * R + row;
    T *to = dx + (tok * rows + head) * p.d + it.a;
    // In a token's last step some rows may not be there, and are zeros: without an epsilon their factor would be infinite, and NaN reach
    // the gains' sums.
    const float last_eps = (s1 - 1) * R + row < rows ? p.eps : 1.f;
    for (int i = s1 - s0; i > 0; i--) {
      cp_async_wait<NRG_STAGES - 2>();
      P2<E> y = unpack2<T>(ring.get(stage, 0));
      const P2<E> x = unpack2<T>(g ? ring.get(stage, 1) : Raw<E>{});
      stage = stage + 1 == NRG_STAGES ? 0 : stage + 1;
      ask();
      if (it.rotates) y = turned<E, I>(y, turn);
      if (g) {
        const P2<E> gain = unpack2<T>(gain_raw);
        P2<E> w;   // t g
#pragma unroll
        for (int e = 0; e < E / 2; e++) w.v[e] = mul_f32x2(y.v[e], gain.v[e]);
        const float ss = group_sum<G>(dot2(x, x)), dot = group_sum<G>(dot2(w, x));
        const float rstd = rsqrtf(fmaf(ss, p.inv_d, i == 1 ? last_eps : p.eps)), mean = dot * rstd * p.inv_d;
        const uint64_t r2 = both(rstd), m2 = both(-mean * rstd);
#pragma unroll
        for (int e = 0; e < E / 2; e++) {
          const uint64_t unit2 = mul_f32x2(x.v[e], r2);
          dg.v[e] = fma_f32x2(y.v[e], unit2, dg.v[e]);
          y.v[e] = fma_f32x2(unit2, m2, mul_f32x2(w.v[e], r2));
        }
      }
      if (head < rows && it.there) store_item(to, ab, pack2<T>(y));
      head += R;
      to += R * p.d;
    }
  }
  if (!partial) return;
  if (it.there) {
#pragma unroll
    for (int i = 0; i < E / 2; i++) {
      float lo, hi;
      unpack_f32x2(dg.v[i], lo, hi);
      float *s = sums[warp * R + row] + (i < E / 4 ? it.a : it.b - E / 2) + 2 * i;
      s[0] = lo;
      s[1] = hi;
    }
  }
  __syncthreads();
  for (int c = tid; c < p.d; c += NRG_THREADS) {
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < GROUPS; r++) s += sums[r][c];
    partial[(size_t)blockIdx.x * p.d + c] = s;
  }
}

// d_g = the blocks' partial sums: 32 columns a block, 32 rows of threads over the partials (a chain of latencies: eight rows
// took 6 us longer for 444 partials)
__global__ void __launch_bounds__(1024)
norm_rope_gains_kernel(const float *__restrict__ partial, int q_blocks, int k_blocks, int d, float *d_g_q, float *d_g_k) {
  __shared__ float sums[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x, w = blockIdx.y;
  float *out = w ? d_g_k : d_g_q;
  pdl_wait();
  if (!out) return;
  const float *from = partial + (w ? (size_t)q_blocks * d : 0);
  const int n = w ? k_blocks : q_blocks;
  float s = 0.f;
  if (c < d) {
#pragma unroll 16
    for (int b = y; b < n; b += 32) s += from[(size_t)b * d + c];
  }
  sums[y][x] = s;
  __syncthreads();
  s = sums[x][y];   // warp y: column y, a lane for every row of threads
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (x == 0 && blockIdx.x * 32 + y < d) out[blockIdx.x * 32 + y] = s;
}

bool aligned16p(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

bool fits32(int64_t stride) { return stride > -(1ll << 31) && stride < (1ll << 31); }

bool rope_args_ok(const locret_rope_args &a) {
  if (a.n_tok < 0 || a.n_q_heads < 1 || a.n_kv_heads < 1 || a.n_q_heads > 65536 || a.n_kv_heads > 65536) return false;
  if (a.head_dim < 8 || a.head_dim > 256 || a.head_dim % 8 || a.rot < 0 || a.rot > a.head_dim || a.rot % 8) return false;
  if (a.dtype != LOCRET_BF16 && a.dtype != LOCRET_FP16) return false;
  if (a.n_tok && a.rot && (!a.positions || !a.turns)) return false;
  if ((a.q_token | a.q_head | a.k_token | a.k_head | a.v_token | a.v_head | a.q_out_token | a.q_out_head | a.k_out_token |
       a.k_out_head) & 7)
    return false;
  if (!fits32(a.q_head) || !fits32(a.k_head) || !fits32(a.v_head) || !fits32(a.q_out_head) || !fits32(a.k_out_head)) return false;
  return aligned16p(a.q) && aligned16p(a.k) && aligned16p(a.v) && aligned16p(a.q_out) && aligned16p(a.k_out) &&
         aligned16p(a.g_q) && aligned16p(a.g_k) && a.eps >= 0.f;
}

NormRope device_args(const locret_rope_args &a) {
  NormRope p = {};
  p.q = a.q; p.k = a.k; p.v = a.v; p.g_q = a.g_q; p.g_k = a.g_k; p.q_out = a.q_out; p.k_out = a.k_out;
  p.q_token = a.q_token; p.k_token = a.k_token; p.v_token = a.v_token;
  p.q_out_token = a.q_out_token; p.k_out_token = a.k_out_token;
  p.q_head = (int)a.q_head; p.k_head = (int)a.k_head; p.v_head = (int)a.v_head;
  p.q_out_head = (int)a.q_out_head; p.k_out_head = (int)a.k_out_head;
  p.positions = a.positions; p.turns = a.turns; p.slots = a.slots; p.status = a.status;
  p.n_tok = a.n_tok; p.h = a.n_q_heads; p.h_kv = a.n_kv_heads; p.d = a.head_dim; p.rot = a.rot;
  p.factor = a.factor; p.eps = a.eps; p.inv_d = 1.0f / (float)a.head_dim;
  return p;
}

// How many warps divide a token's steps: enough that the tokens make NR_PER_SM warps for each SM, one step each at most.
constexpr int NR_PER_SM = 16;
int slices_of(int n_tok, int steps) {
  const long long want = ((long long)sm_count_of_current_device() * NR_PER_SM + n_tok - 1) / (n_tok < 1 ? 1 : n_tok);
  return want < 1 ? 1 : want > steps ? steps : (int)want;
}

template <typename T, int E, int G, int I>
cudaError_t launch_forward(const NormRope &p, cudaStream_t st) {
  constexpr int R = 32 / G;
  const int slices = slices_of(p.n_tok, (p.h + R - 1) / R + (p.pages.k ? 2 : 1) * ((p.h_kv + R - 1) / R));
  const long long units = (long long)p.n_tok * slices;
  norm_rope_kernel<T, E, G, I><<<(unsigned)((units + NR_WARPS - 1) / NR_WARPS), NR_THREADS, 0, st>>>(p, slices);
  return cudaGetLastError();
}

// The gradients' grid: at most NRG_PER_SM blocks an SM, dealt in proportion to the rows.
constexpr int NRG_PER_SM = 3;
int grad_blocks() { return sm_count_of_current_device() * NRG_PER_SM; }

template <typename T, int E, int G, int I>
cudaError_t launch_backward(const NormRope &p, void *d_q, void *d_k, float *d_g_q, float *d_g_k, float *partial, cudaStream_t st) {
  constexpr int R = 32 / G;
  const int q_steps = (p.h + R - 1) / R, k_steps = (p.h_kv + R - 1) / R, all = grad_blocks();
  int for_q = (int)((long long)all * q_steps / (q_steps + k_steps));
  for_q = for_q < 1 ? 1 : for_q >= all ? all - 1 : for_q;
  auto part = [&](int steps, int most) {
    Part x = {most, slices_of(p.n_tok, steps)};
    const long long blocks = ((long long)p.n_tok * x.slices + NRG_WARPS - 1) / NRG_WARPS;
    if (blocks < x.blocks) x.blocks = (int)blocks;
    return x;
  };
  const Part q = part(q_steps, for_q), k = part(k_steps, all - for_q);
  if (p.n_tok > 0) {
    norm_rope_grad_kernel<T, E, G, I><<<q.blocks + k.blocks, NRG_THREADS, 0, st>>>(p, q, k, static_cast<T *>(d_q),
                                                                                 static_cast<T *>(d_k), partial);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if (!partial) return cudaSuccess;
  return launch_kernel(norm_rope_gains_kernel, dim3((p.d + 31) / 32, 2), dim3(1024), 0, st, true, (const float *)partial, q.blocks,
                       k.blocks, p.d, d_g_q, d_g_k);
}

// call<T, E, G, I> for the type, elements per item, lanes per row and pairing
#define NR_DISPATCH(call)                                                                          \
  [&]() -> cudaError_t {                                                                           \
    auto by_pairs = [&](auto t, auto e, auto g) -> cudaError_t {                                   \
      using T = decltype(t);                                                                       \
      constexpr int E = decltype(e)::value, G = decltype(g)::value;                                \
      if (args->interleaved) { constexpr int I = 1; return call; }                                 \
      constexpr int I = 0;                                                                         \
      return call;                                                                                 \
    };                                                                                             \
    auto by_lanes = [&](auto t) -> cudaError_t {                                                   \
      if (p.d % 16 == 0 && p.rot % 16 == 0) {                                                      \
        if (p.d <= 64) return by_pairs(t, Int<16>(), Int<4>());                                    \
        if (p.d <= 128) return by_pairs(t, Int<16>(), Int<8>());                                   \
        return by_pairs(t, Int<16>(), Int<16>());                                                  \
      }                                                                                            \
      if (p.d <= 128) return by_pairs(t, Int<8>(), Int<16>());                                     \
      return by_pairs(t, Int<8>(), Int<32>());                                                     \
    };                                                                                             \
    return args->dtype == LOCRET_BF16 ? by_lanes(bf16()) : by_lanes(__half());                     \
  }()
template <int N> using Int = std::integral_constant<int, N>;

}  // namespace
}  // namespace locret

using namespace locret;

extern "C" int locret_norm_rope(const locret_rope_args *args, void *stream) {
  if (!args || !rope_args_ok(*args)) return LOCRET_ERR_INVALID;
  if (args->n_tok && (!args->q || !args->k || !args->q_out)) return LOCRET_ERR_INVALID;
  if (args->pages) {
    const locret_pages &g = *args->pages;
    if (!pages_ok(g) || g.dtype != args->dtype || g.n_kv_heads != args->n_kv_heads || g.head_dim != args->head_dim ||
        (args->n_tok && (!args->v || !args->slots)))
      return LOCRET_ERR_INVALID;
  } else if (args->v || args->slots || (args->n_tok && !args->k_out)) {
    return LOCRET_ERR_INVALID;
  }
  if (args->n_tok == 0) return LOCRET_OK;
  NormRope p = device_args(*args);
  if (args->pages) p.pages = page_view(*args->pages);
  const cudaError_t e = NR_DISPATCH((launch_forward<T, E, G, I>(p, (cudaStream_t)stream)));
  if (e != cudaSuccess) { cudaGetLastError(); return LOCRET_ERR_CUDA; }
  return LOCRET_OK;
}

extern "C" int locret_norm_rope_grad_workspace(int32_t head_dim, int64_t *bytes) {
  if (!bytes || head_dim < 8 || head_dim > 256 || head_dim % 8) return LOCRET_ERR_INVALID;
  *bytes = (int64_t)grad_blocks() * head_dim * sizeof(float);
  return LOCRET_OK;
}

extern "C" int locret_norm_rope_grad(const locret_rope_args *args, void *d_q, void *d_k, float *d_g_q, float *d_g_k,
                                     void *workspace, int64_t workspace_bytes, void *stream) {
  if (!args || !rope_args_ok(*args)) return LOCRET_ERR_INVALID;
  if (args->n_tok && (!args->q_out || !args->k_out || !d_q || !d_k)) return LOCRET_ERR_INVALID;
  if (!aligned16p(d_q) || !aligned16p(d_k)) return LOCRET_ERR_INVALID;
  if ((args->g_q != nullptr) != (d_g_q != nullptr) || (args->g_k != nullptr) != (d_g_k != nullptr)) return LOCRET_ERR_INVALID;
  if (args->n_tok && ((args->g_q && !args->q) || (args->g_k && !args->k))) return LOCRET_ERR_INVALID;
  const bool norm = d_g_q || d_g_k;
  int64_t need = 0;
  locret_norm_rope_grad_workspace(args->head_dim, &need);
  if (norm && (!workspace || !aligned16p(workspace))) return LOCRET_ERR_INVALID;
  if (norm && workspace_bytes < need) return LOCRET_ERR_CAPACITY;
  const cudaStream_t st = (cudaStream_t)stream;
  const NormRope p = device_args(*args);
  float *partial = norm ? static_cast<float *>(workspace) : nullptr;
  const cudaError_t e = NR_DISPATCH((launch_backward<T, E, G, I>(p, d_q, d_k, d_g_q, d_g_k, partial, st)));
  if (e != cudaSuccess) { cudaGetLastError(); return LOCRET_ERR_CUDA; }
  return LOCRET_OK;
}
