// Norms of queries and keys for each head, rotation, cache append; and the gradients.  Bound by memory: every element is read
// and written once.
#include <type_traits>

#include "../../include/locret.h"
#include "common.cuh"
#include "paged.cuh"

namespace locret {
namespace {

constexpr int NR_THREADS = 256, NR_MAX_TOKENS = 4;

struct NormRope {
  const void *q, *k, *v, *g_q, *g_k;
  void *q_out, *k_out;
  long long q_token, q_head, k_token, k_head, v_token, v_head, q_out_token, q_out_head, k_out_token, k_out_head;
  const int32_t *positions;
  const uint64_t *turns;
  const int64_t *slots;
  int32_t *status;
  PageView pages;
  int n_tok, h, h_kv, d, rot, interleaved, tokens;   // tokens: per block
  float factor, eps;
};

// Cosine and sine of position * turns / 2^64 turns.  The product's low 64 bits are the exact fraction of a turn at every
// position; its upper 32 bits, as a signed number, are the angle to 2^-32 turns.
__device__ __forceinline__ float2 cos_sin(uint64_t turns, int position, float factor) {
  const int32_t top = (int32_t)((turns * (uint64_t)(int64_t)position) >> 32);
  float s, c;
  sincospif((float)top * (1.0f / 2147483648.0f), &s, &c);
  return make_float2(c * factor, s * factor);
}

// A row (one head of one token) is d / 8 items of eight elements, one for each lane of a group.  Item j < rot / 8 holds pairs
// 4j .. 4j+3 whole - with half rotation, four elements of either half - so a rotation needs no other lane; two 8-byte accesses
// an item, neighbouring lanes next to each other.
struct Item {
  int a, b;       // offsets of its two runs of four elements
  bool rotates, there;
};
__device__ __forceinline__ Item item_of(int j, int d, int rot, int interleaved) {
  Item it;
  it.there = j * 8 < d;
  it.rotates = j * 8 < rot;
  it.a = it.rotates && !interleaved ? 4 * j : 8 * j;
  it.b = it.rotates && !interleaved ? rot / 2 + 4 * j : 8 * j + 4;
  return it;
}

template <typename T>
__device__ __forceinline__ void unpack8(uint2 a, uint2 b, float (&x)[8]) {
  const float2 f0 = Half2<T>::unpack(a.x), f1 = Half2<T>::unpack(a.y), f2 = Half2<T>::unpack(b.x), f3 = Half2<T>::unpack(b.y);
  x[0] = f0.x; x[1] = f0.y; x[2] = f1.x; x[3] = f1.y;
  x[4] = f2.x; x[5] = f2.y; x[6] = f3.x; x[7] = f3.y;
}
template <typename T>
__device__ __forceinline__ void pack8(const float (&x)[8], uint2 &a, uint2 &b) {
  a = make_uint2(Half2<T>::pack(x[0], x[1]), Half2<T>::pack(x[2], x[3]));
  b = make_uint2(Half2<T>::pack(x[4], x[5]), Half2<T>::pack(x[6], x[7]));
}

template <typename T>
__device__ __forceinline__ void load8(const T *row, const Item &it, uint2 &a, uint2 &b) {
  a = b = make_uint2(0, 0);
  if (it.there) {
    a = *reinterpret_cast<const uint2 *>(row + it.a);
    b = *reinterpret_cast<const uint2 *>(row + it.b);
  }
}
template <typename T>
__device__ __forceinline__ void store8(T *row, const Item &it, uint2 a, uint2 b) {
  if (it.there) {
    *reinterpret_cast<uint2 *>(row + it.a) = a;
    *reinterpret_cast<uint2 *>(row + it.b) = b;
  }
}

// rotation of an item's four pairs by (c, s), or back with (c, -s)
__device__ __forceinline__ void rotate8(float (&x)[8], const float2 (&cs)[4], int interleaved) {
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const int ia = interleaved ? 2 * i : i, ib = interleaved ? 2 * i + 1 : i + 4;
    const float a = x[ia], b = x[ib];
    x[ia] = a * cs[i].x - b * cs[i].y;
    x[ib] = a * cs[i].y + b * cs[i].x;
  }
}

template <int G>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// G lanes a row (8, 16 or 32: the power of two that covers d / 8).  A block takes `tokens` tokens and all their heads.
template <typename T, int G, int I>
__global__ void __launch_bounds__(NR_THREADS) norm_rope_kernel(const __grid_constant__ NormRope p) {
  constexpr int ROWS = NR_THREADS / G;
  __shared__ float2 cs_s[NR_MAX_TOKENS][128];
  const int tid = threadIdx.x, j = tid % G, row0 = tid / G;
  const int t0 = blockIdx.x * p.tokens, nt = min(p.tokens, p.n_tok - t0), half = p.rot / 2;
  for (int x = tid; x < nt * half; x += NR_THREADS) {
    const int t = x / half, i = x - t * half;
    cs_s[t][i] = cos_sin(p.turns[i], p.positions[t0 + t], p.factor);
  }
  const Item it = item_of(j, p.d, p.rot, I);
  float gain[2][8];
#pragma unroll
  for (int w = 0; w < 2; w++) {
    const T *g = static_cast<const T *>(w ? p.g_k : p.g_q);
    uint2 a = make_uint2(0, 0), b = a;
    if (g) load8(g, it, a, b);
    unpack8<T>(a, b, gain[w]);
  }
  __syncthreads();
  const int n_rows = p.h + p.h_kv + (p.pages.k ? p.h_kv : 0);
  for (int t = 0; t < nt; t++) {
    const long long tok = t0 + t;
    float2 cs[4] = {};
    if (it.rotates) {
#pragma unroll
      for (int i = 0; i < 4; i++) cs[i] = cs_s[t][4 * j + i];
    }
    long long at = -1;   // the token's place in the pool (key and value of head 0)
    if (p.pages.k) {
      const int64_t slot = p.slots[tok];
      if (slot >= 0) {
        const int64_t page = slot / p.pages.page_size;
        if (page < p.pages.n_pages) at = page * p.pages.page_stride + (slot - page * p.pages.page_size) * p.pages.token_stride;
        else if (tid == 0) report(p.status, LOCRET_ERR_INVALID);
      }
    }
    for (int r = row0; r - row0 < n_rows; r += ROWS) {   // (the same number of turns for every lane of a warp)
      const int kind = r < p.h ? 0 : r < p.h + p.h_kv ? 1 : r < n_rows ? 2 : 3, head = r - (kind == 0 ? 0 : kind == 1 ? p.h : p.h + p.h_kv);
      uint2 a = make_uint2(0, 0), b = a;
      if (kind == 0) load8(static_cast<const T *>(p.q) + tok * p.q_token + head * p.q_head, it, a, b);
      if (kind == 1) load8(static_cast<const T *>(p.k) + tok * p.k_token + head * p.k_head, it, a, b);
      if (kind == 2) load8(static_cast<const T *>(p.v) + tok * p.v_token + head * p.v_head, it, a, b);
      float x[8];
      unpack8<T>(a, b, x);
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 8; e++) ss = fmaf(x[e], x[e], ss);
      ss = group_sum<G>(ss);
      if (kind < 2) {
        if (kind == 0 ? p.g_q != nullptr : p.g_k != nullptr) {
          const float rstd = rsqrtf(ss / p.d + p.eps);
#pragma unroll
          for (int e = 0; e < 8; e++) x[e] = x[e] * rstd * gain[kind][e];
        }
        if (it.rotates) rotate8(x, cs, I);
        pack8<T>(x, a, b);
      }
      if (kind == 0) store8(static_cast<T *>(p.q_out) + tok * p.q_out_token + head * p.q_out_head, it, a, b);
      if (kind == 1 && p.k_out) store8(static_cast<T *>(p.k_out) + tok * p.k_out_token + head * p.k_out_head, it, a, b);
      if ((kind == 1 || kind == 2) && at >= 0)
        store8(static_cast<T *>(kind == 1 ? p.pages.k : p.pages.v) + at + head * p.pages.head_stride, it, a, b);
    }
  }
}

// ---------------------------------------------------------------- gradients
//   t = R^T dy,  n = x rstd,  d_g = sum t n,  dx = rstd (t g - n mean(t g n));   without a norm dx = t
// A persistent grid: a block adds up t n of its tokens in registers and writes one partial sum per gain; a second kernel adds
// those, in the order of the blocks.
constexpr int NRG_MAX_BLOCKS = 148 * 4;

template <typename T, int G, int I>
__global__ void __launch_bounds__(NR_THREADS)
norm_rope_grad_kernel(const __grid_constant__ NormRope p, T *d_q, T *d_k, float *partial) {
  constexpr int ROWS = NR_THREADS / G;
  __shared__ float2 cs_s[128];
  __shared__ float sums[ROWS][G * 8];
  const int tid = threadIdx.x, j = tid % G, row0 = tid / G, half = p.rot / 2;
  const Item it = item_of(j, p.d, p.rot, I);
  float gain[2][8], dg[2][8] = {};
#pragma unroll
  for (int w = 0; w < 2; w++) {
    const T *g = static_cast<const T *>(w ? p.g_k : p.g_q);
    uint2 a = make_uint2(0, 0), b = a;
    if (g) load8(g, it, a, b);
    unpack8<T>(a, b, gain[w]);
  }
  const int n_rows = p.h + p.h_kv;
  for (long long tok = blockIdx.x; tok < p.n_tok; tok += gridDim.x) {
    __syncthreads();
    for (int i = tid; i < half; i += NR_THREADS) cs_s[i] = cos_sin(p.turns[i], p.positions[tok], p.factor);
    __syncthreads();
    float2 cs[4] = {};
    if (it.rotates) {
#pragma unroll
      for (int i = 0; i < 4; i++) { cs[i] = cs_s[4 * j + i]; cs[i].y = -cs[i].y; }
    }
    for (int r = row0; r - row0 < n_rows; r += ROWS) {
      const int kind = r < p.h ? 0 : r < n_rows ? 1 : 2, head = r - (kind ? p.h : 0);
      const bool norm = kind == 0 ? p.g_q != nullptr : kind == 1 && p.g_k != nullptr;
      uint2 a = make_uint2(0, 0), b = a, xa = a, xb = a;
      if (kind == 0) {
        load8(static_cast<const T *>(p.q_out) + tok * p.q_out_token + head * p.q_out_head, it, a, b);
        if (norm) load8(static_cast<const T *>(p.q) + tok * p.q_token + head * p.q_head, it, xa, xb);
      }
      if (kind == 1) {
        load8(static_cast<const T *>(p.k_out) + tok * p.k_out_token + head * p.k_out_head, it, a, b);
        if (norm) load8(static_cast<const T *>(p.k) + tok * p.k_token + head * p.k_head, it, xa, xb);
      }
      float y[8], x[8];
      unpack8<T>(a, b, y);
      unpack8<T>(xa, xb, x);
      if (it.rotates) rotate8(y, cs, I);
      float ss = 0.f, dot = 0.f;   // sum x^2, sum t g x
#pragma unroll
      for (int e = 0; e < 8; e++) {
        ss = fmaf(x[e], x[e], ss);
        dot = fmaf(y[e] * gain[kind & 1][e], x[e], dot);
      }
      ss = group_sum<G>(ss);
      dot = group_sum<G>(dot);
      if (norm) {
        const float rstd = rsqrtf(ss / p.d + p.eps), mean = dot * rstd / p.d;
#pragma unroll
        for (int e = 0; e < 8; e++) {
          const float n = x[e] * rstd;
          dg[0][e] += kind == 0 ? y[e] * n : 0.f;
          dg[1][e] += kind == 1 ? y[e] * n : 0.f;
          y[e] = rstd * (y[e] * gain[kind & 1][e] - n * mean);
        }
      }
      pack8<T>(y, a, b);
      if (kind == 0) store8(d_q + (tok * p.h + head) * p.d, it, a, b);
      if (kind == 1) store8(d_k + (tok * p.h_kv + head) * p.d, it, a, b);
    }
  }
  if (!partial) return;
#pragma unroll
  for (int w = 0; w < 2; w++) {
    __syncthreads();
    if (it.there) {
#pragma unroll
      for (int e = 0; e < 8; e++) sums[row0][(e < 4 ? it.a : it.b) + (e & 3)] = dg[w][e];
    }
    __syncthreads();
    for (int c = tid; c < p.d; c += NR_THREADS) {
      float s = 0.f;
#pragma unroll
      for (int r = 0; r < ROWS; r++) s += sums[r][c];
      partial[((size_t)blockIdx.x * 2 + w) * p.d + c] = s;
    }
  }
}

// d_g = the blocks' partial sums: 32 columns a block, eight rows of threads over the partials
__global__ void __launch_bounds__(256)
norm_rope_gains_kernel(const float *__restrict__ partial, int n_blocks, int d, float *d_g_q, float *d_g_k) {
  __shared__ float sums[8][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x, w = blockIdx.y;
  float *out = w ? d_g_k : d_g_q;
  if (!out) return;
  float s = 0.f;
  if (c < d)
    for (int b = y; b < n_blocks; b += 8) s += partial[((size_t)b * 2 + w) * d + c];
  sums[y][x] = s;
  __syncthreads();
  if (y == 0 && c < d) {
    s = 0.f;
#pragma unroll
    for (int r = 0; r < 8; r++) s += sums[r][x];
    out[c] = s;
  }
}

bool aligned16p(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

bool rope_args_ok(const locret_rope_args &a) {
  if (a.n_tok < 0 || a.n_q_heads < 1 || a.n_kv_heads < 1 || a.n_q_heads > 65536 || a.n_kv_heads > 65536) return false;
  if (a.head_dim < 8 || a.head_dim > 256 || a.head_dim % 8 || a.rot < 0 || a.rot > a.head_dim || a.rot % 8) return false;
  if (a.dtype != LOCRET_BF16 && a.dtype != LOCRET_FP16) return false;
  if (a.n_tok && a.rot && (!a.positions || !a.turns)) return false;
  if ((a.q_token | a.q_head | a.k_token | a.k_head | a.v_token | a.v_head | a.q_out_token | a.q_out_head | a.k_out_token |
       a.k_out_head) & 7)
    return false;
  return aligned16p(a.q) && aligned16p(a.k) && aligned16p(a.v) && aligned16p(a.q_out) && aligned16p(a.k_out) &&
         aligned16p(a.g_q) && aligned16p(a.g_k) && a.eps >= 0.f;
}

NormRope device_args(const locret_rope_args &a) {
  NormRope p = {};
  p.q = a.q; p.k = a.k; p.v = a.v; p.g_q = a.g_q; p.g_k = a.g_k; p.q_out = a.q_out; p.k_out = a.k_out;
  p.q_token = a.q_token; p.q_head = a.q_head; p.k_token = a.k_token; p.k_head = a.k_head;
  p.v_token = a.v_token; p.v_head = a.v_head;
  p.q_out_token = a.q_out_token; p.q_out_head = a.q_out_head; p.k_out_token = a.k_out_token; p.k_out_head = a.k_out_head;
  p.positions = a.positions; p.turns = a.turns; p.slots = a.slots; p.status = a.status;
  p.n_tok = a.n_tok; p.h = a.n_q_heads; p.h_kv = a.n_kv_heads; p.d = a.head_dim; p.rot = a.rot; p.interleaved = a.interleaved;
  p.factor = a.factor; p.eps = a.eps;
  return p;
}

template <typename T, int G, int I>
cudaError_t launch_forward(const NormRope &p, cudaStream_t st) {
  norm_rope_kernel<T, G, I><<<(p.n_tok + p.tokens - 1) / p.tokens, NR_THREADS, 0, st>>>(p);
  return cudaGetLastError();
}

template <typename T, int G, int I>
cudaError_t launch_backward(const NormRope &p, void *d_q, void *d_k, float *partial, int blocks, cudaStream_t st) {
  norm_rope_grad_kernel<T, G, I><<<blocks, NR_THREADS, 0, st>>>(p, static_cast<T *>(d_q), static_cast<T *>(d_k), partial);
  return cudaGetLastError();
}

// f<T, G, I>(...) for the type, lanes per row and pairing
#define NR_DISPATCH(call)                                                                          \
  [&]() -> cudaError_t {                                                                           \
    auto by_pairs = [&](auto t, auto g) -> cudaError_t {                                           \
      using T = decltype(t);                                                                       \
      constexpr int G = decltype(g)::value;                                                        \
      if (p.interleaved) { constexpr int I = 1; return call; }                                     \
      constexpr int I = 0;                                                                         \
      return call;                                                                                 \
    };                                                                                             \
    auto by_lanes = [&](auto t) -> cudaError_t {                                                   \
      if (p.d <= 64) return by_pairs(t, std::integral_constant<int, 8>());                         \
      if (p.d <= 128) return by_pairs(t, std::integral_constant<int, 16>());                       \
      return by_pairs(t, std::integral_constant<int, 32>());                                       \
    };                                                                                             \
    return args->dtype == LOCRET_BF16 ? by_lanes(bf16()) : by_lanes(__half());                     \
  }()

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
  p.tokens = 1;
  const cudaError_t e = NR_DISPATCH((launch_forward<T, G, I>(p, (cudaStream_t)stream)));
  if (e != cudaSuccess) { cudaGetLastError(); return LOCRET_ERR_CUDA; }
  return LOCRET_OK;
}

extern "C" int locret_norm_rope_grad_workspace(int32_t head_dim, int64_t *bytes) {
  if (!bytes || head_dim < 8 || head_dim > 256 || head_dim % 8) return LOCRET_ERR_INVALID;
  *bytes = (int64_t)NRG_MAX_BLOCKS * 2 * head_dim * sizeof(float);
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
  const int blocks = p.n_tok < NRG_MAX_BLOCKS ? p.n_tok : NRG_MAX_BLOCKS;
  float *partial = norm ? static_cast<float *>(workspace) : nullptr;
  if (blocks) {
    const cudaError_t e = NR_DISPATCH((launch_backward<T, G, I>(p, d_q, d_k, partial, blocks, st)));
    if (e != cudaSuccess) { cudaGetLastError(); return LOCRET_ERR_CUDA; }
  }
  if (norm) {
    norm_rope_gains_kernel<<<dim3((p.d + 31) / 32, 2), 256, 0, st>>>(partial, blocks, p.d, d_g_q, d_g_k);
    if (cudaGetLastError() != cudaSuccess) return LOCRET_ERR_CUDA;
  }
  return LOCRET_OK;
}
