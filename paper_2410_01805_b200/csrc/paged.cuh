// What the calls on pages share: the pool as a kernel sees it, 16-bit types, and the host's checks.
#pragma once

#include "../../include/locret.h"
#include "common.cuh"

namespace locret {

// n / d for 0 <= n < 2^31: n * ceil(2^(31 + s) / d) >> (31 + s) with s = ceil(log2 d).  Exact: the factor exceeds 2^(31 + s) / d by
// less than 1, so the quotient by less than n * 2^-(31 + s) < 2^-s <= 1 / d, which does not reach the next whole number.
struct FastDiv {
  uint32_t mul, shift;
  FastDiv() = default;
  explicit FastDiv(uint32_t d) {
    uint32_t s = 0;
    while ((1ull << s) < d) s++;
    shift = 31 + s;
    mul = (uint32_t)(((1ull << shift) + d - 1) / d);
  }
  __device__ __forceinline__ int div(int n) const { return (int)(((uint64_t)(uint32_t)n * mul) >> shift); }
};

struct PageView {
  void *k, *v;
  long long page_stride, head_stride, token_stride;   // elements
  int n_pages, page_size;
  FastDiv by_size;
};

inline PageView page_view(const locret_pages &p) {
  return PageView{p.k, p.v, p.page_stride, p.head_stride, p.token_stride, p.n_pages, p.page_size, FastDiv(p.page_size)};
}

inline bool pages_ok(const locret_pages &p) {
  return p.k && p.v && !((reinterpret_cast<uintptr_t>(p.k) | reinterpret_cast<uintptr_t>(p.v)) & 15u) && p.n_pages >= 1 &&
         p.page_size >= 1 && p.n_kv_heads >= 1 && p.head_dim >= 8 && (p.dtype == LOCRET_BF16 || p.dtype == LOCRET_FP16) &&
         p.page_stride >= 0 && p.head_stride >= 0 && p.token_stride >= 0 &&
         !((p.page_stride | p.head_stride | p.token_stride) & 7);
}

// what a kernel found wrong, into the caller's word
__device__ __forceinline__ void report(int32_t *status, int code) {
  if (status) atomicMin(status, code);
}

// the two 16-bit types
template <typename T> struct Half2;
template <> struct Half2<bf16> {
  static __device__ __forceinline__ float2 unpack(uint32_t v) {
    return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&v));
  }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_bf16(lo, hi); }
};
template <> struct Half2<__half> {
  static __device__ __forceinline__ float2 unpack(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2 *>(&v)); }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
  }
};

cudaError_t launch_export_pages(const bf16 *k_rot, const bf16 *v, const int32_t *rank, int h_kv, int d, int cap, int len,
                                int ranked_len, const int32_t *table, const locret_pages &pages, int32_t *status, cudaStream_t st);

}  // namespace locret
