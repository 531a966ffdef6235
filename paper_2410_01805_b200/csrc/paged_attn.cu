// Attention of one new token per request over pages, divided over the GPU and joined.
//
// Bound by memory: every visible key and value is read once, 4 d bytes of each for 4 g d operations.  So the kernel is a
// stream of asynchronous copies with the arithmetic hidden behind it:
//  * The visible keys of every (request, KV head) are cut into steps (16 per warp), and all steps of the batch, one after the other,
//    form a line that is cut into equal parts, one for each block of a persistent grid: lengths may differ as they like, and
//    one long request fills the GPU as well as many short ones.  Every block finds its part by summing the lengths itself.
//  * A warp takes 16 keys of each step and has a ring of stages of its own, filled by its own copies: no barrier of the block
//    stands in the loop.  Keys are the m side of m16n8k16 tiles and the heads of a group (eight; sixteen in two tiles) the n
//    side: S^T = K Q^T, O^T = V^T P^T, with an 8 x 8 transpose of P in between.
//  * The softmax keeps a running scale per head that is raised only when a weight would exceed 2^8, fp16 2^4 (then the 16 keys' maximum
//    is found and the sums are rescaled): most steps need one vote in place of the reductions.
//  * The warps of a block meet at the end of a (request, KV head); where the line was cut inside one, the blocks leave partial
//    results that a second kernel joins, in the order of the blocks.
#include <float.h>
#include <math.h>

#include "../../include/locret.h"
#include "common.cuh"
#include "paged.cuh"

namespace locret {
namespace {

// Warps of a block, stages of a warp's ring, blocks of an SM, and whether there are two buffers in which the warps meet.  What the
// loop waits for is its own chain of instructions, so more warps do more than more stages, as far as shared memory goes (four
// warps with three stages each, then these: two KV heads of 64, 1.03 GB: 192, 171 us; 32 of 96, a window, 1.05 GB: 181, 174; eight
// of 128, one request, 4.1 GB: 655, 630).  With sixteen heads a block, five warps of two stages take 122 us for 109.
template <int D, int NT> struct PaCfg { static constexpr int WARPS = 4, STAGES = 3, PER_SM = 2; static constexpr bool TWO = false; };
template <> struct PaCfg<128, 1> { static constexpr int WARPS = 5, STAGES = 2, PER_SM = 2; static constexpr bool TWO = true; };
template <> struct PaCfg<96, 1> { static constexpr int WARPS = 5, STAGES = 2, PER_SM = 2; static constexpr bool TWO = true; };
template <> struct PaCfg<64, 1> { static constexpr int WARPS = 7, STAGES = 2, PER_SM = 2; static constexpr bool TWO = true; };
constexpr int PA_WHOLE = 6;        // steps up to which items are not divided (see launch)
// A key's weight is 1 where it sets the running scale, and at most 2^MOST before the scale is raised.  The second product takes it,
// times UP, as the sum of two 16-bit numbers.  bf16 has the range for any of them, and 16 bits of each (2^-17, against 2^-8 for the
// output's rounding) cost two products; more would cost three.  fp16 has 22 bits (2^-23) of a number from 2^-2 on, and of a smaller one
// what lies above 2^-25: so its weights are carried as high as they can be, and what is lost of a key is at most 2^-36 of the largest
// key's weight (2^-25 with UP 1 and MOST 8; the same time: 24 requests, a window of 4096, 32 heads of 96, 177 us).  The sums of
// weights go without UP: as 11 in the exponent it cost no product, but each weight, and the logarithm of the sum, 2^-21.
template <typename T> struct PaWeight { static constexpr float MOST = 8.f, UP = 1.f; };
template <> struct PaWeight<__half> { static constexpr float MOST = 4.f, UP = 2048.f; };

template <typename T>
__device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16<bf16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16<__half>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}

__device__ __forceinline__ float exp2_fast(float x) {   // (results below 2^-126 are 0)
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

struct PagedAttn {
  const void *q;
  void *out;
  float *lse, *part;       // part: [block][2] partial results of HB heads: sums [HB][d], then (scale, sum) [HB][2]
  int4 *rec;               // [block]: x = request whose part begins in the block and does not end there (-1: none), y = its
                           // item, z = 1 if the block's first part goes on behind it, 2 if it ends there (0: none)
  const int32_t *table, *lens;
  int32_t *status;
  const uint4 *k, *v;      // the pool; places in it in units of 16 bytes, 32 bits (one exchange and one product instead of several)
  uint32_t page_stride, head_stride, token_stride;
  int n_pages, page_size;
  FastDiv by_size;
  long long q_req, q_head, out_req, out_head, table_stride;
  int width, n_req, h, h_kv, groups, window, sinks;   // groups: blocks of heads per KV head
  int whole;                                           // no item is divided (none is long): nothing to join
  float scale_log2;
};

// A request's visible keys, numbered 0 .. n-1: key i is i for i < sinks, else i + shift.
struct Visible {
  int n, shift, sinks;
  __device__ __forceinline__ int key(int i) const { return i < sinks ? i : i + shift; }
  // (an empty request has one step, to write zeros)
  template <int STEP> __device__ __forceinline__ int steps() const { return n > 0 ? (n - 1) / STEP + 1 : 1; }
  template <int WARPS> __device__ __forceinline__ int steps(bool solo) const { return solo ? steps<16>() : steps<16 * WARPS>(); }
};
__device__ __forceinline__ int clamped_len(const PagedAttn &a, int r) {
  const int n = __ldg(a.lens + r);
  return max(0, (int)min((long long)n, (long long)a.width * a.page_size));
}
__device__ __forceinline__ Visible visible_of(const PagedAttn &a, int len) {
  Visible v = {len, 0, 0};
  if (a.window > 0) {
    const int start = max(a.sinks, len - a.window);
    v.sinks = a.sinks;
    v.shift = start - a.sinks;
    v.n = min(len, a.sinks) + max(0, len - start);
  }
  return v;
}

// A place in the line: step `tile` of KV head m and block of heads hg of request r.
template <int WARPS>
struct Cursor {
  int r, m, hg, tile, steps, next_len;   // next_len: of the request behind, on its way
  uint32_t head_at;                      // where head m begins in a page
  const int32_t *row;                    // the request's pages
  Visible v;
  bool solo;
  __device__ __forceinline__ void enter(const PagedAttn &a, int request, int len) {
    r = request;
    m = hg = tile = 0;
    head_at = 0;
    row = a.table + r * a.table_stride;
    v = visible_of(a, len);
    steps = v.template steps<WARPS>(solo);
    next_len = clamped_len(a, min(r + 1, a.n_req - 1));
  }
  __device__ __forceinline__ void next(const PagedAttn &a) {
    if (++tile < steps) return;
    tile = 0;
    if (++hg < a.groups) return;
    hg = 0;
    head_at += a.head_stride;
    if (++m < a.h_kv) return;
    enter(a, r + 1, next_len);
  }
};
// (m, hg) in one word, for the records
__device__ __forceinline__ int pack_item(int m, int hg) { return (int)((uint32_t)m | (uint32_t)hg << 16); }
__device__ __forceinline__ int item_m(int item) { return item & 0xffff; }
__device__ __forceinline__ int item_hg(int item) { return (int)((uint32_t)item >> 16); }

// What a block - or, `solo`, a warp - does of the line: n steps from step `into` of request r (in steps of all its items).
// Solo is for many short requests: a warp takes whole items, 16 keys a step, and the warps of a block need not meet, which costs
// an item as much as about two steps.  A warp's share then ends with an item, so it is uneven by the longest of them; the
// other way a block's share ends anywhere.  Taken where that makes the shorter time (413 requests of one or two tokens, eight
// heads of 64: 33 us one way, 14.7 the other; 512 requests of 10 to 400 tokens, eight of 128: 115 and 110).
struct Share {
  int r, n;
  long long into;
  bool solo;
};
template <int WARPS>
__device__ Share find_share(const PagedAttn &a, int items) {
  constexpr int THREADS = WARPS * 32;
  __shared__ long long sums[2][WARPS], found_into[WARPS + 1];
  __shared__ int longest[WARPS], found_r[WARPS + 1];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // every warp by itself for up to 32 requests, else the block
  const bool few = a.n_req <= 32;
  const int at = few ? lane : tid, per = few ? 1 : (a.n_req + THREADS - 1) / THREADS;
  const int r0 = min(a.n_req, at * per), r1 = min(a.n_req, r0 + per);
  long long mine_b = 0, mine_w = 0;   // steps of the thread's requests, for one item, by blocks and by warps
  int most = 0;
  for (int r = r0; r < r1; r++) {
    const int raw = __ldg(a.lens + r), len = clamped_len(a, r);
    if (raw != len && blockIdx.x == 0) report(a.status, LOCRET_ERR_INVALID);
    const Visible v = visible_of(a, len);
    const int w = v.template steps<16>();
    mine_b += v.template steps<16 * WARPS>();
    mine_w += w;
    most = max(most, w);
  }
  long long upto_b = mine_b, upto_w = mine_w;   // with all before it
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, upto_b, o), z = __shfl_up_sync(0xffffffffu, upto_w, o);
    if (lane >= o) { upto_b += y; upto_w += z; }
  }
  most = __reduce_max_sync(0xffffffffu, most);
  long long total_b = __shfl_sync(0xffffffffu, upto_b, 31), total_w = __shfl_sync(0xffffffffu, upto_w, 31);
  if (!few) {
    if (lane == 31) { sums[0][warp] = upto_b; sums[1][warp] = upto_w; longest[warp] = most; }
    if (tid <= WARPS) { found_r[tid] = a.n_req; found_into[tid] = 0; }
    __syncthreads();
    total_b = total_w = 0;
#pragma unroll
    for (int w = 0; w < WARPS; w++) {
      if (w < warp) { upto_b += sums[0][w]; upto_w += sums[1][w]; }
      total_b += sums[0][w];
      total_w += sums[1][w];
      most = max(most, longest[w]);
    }
  }
  total_b *= items;
  total_w *= items;
  const long long n_items = (long long)a.n_req * items, blocks = gridDim.x;
  Share s;
  s.solo = total_w + most * blocks * WARPS < (total_b + 2 * n_items) * WARPS;   // (shares, times the number of warps)
  const long long mine = (s.solo ? mine_w : mine_b) * items, upto = (s.solo ? upto_w : upto_b) * items, total = s.solo ? total_w : total_b;
  // With fewer steps than blocks the first blocks take one each, so that no block between two parts of an item is empty.
  const long long parts = s.solo ? blocks * WARPS : min(blocks, total), first = (long long)blockIdx.x * (s.solo ? WARPS : 1);
  const bool whole = s.solo || a.whole;   // parts end with an item
  const bool narrow = total * parts <= 0xffffffffll;   // (a division of 64 bits is a long way from the first request for a key)
  auto cut = [&](long long part) {
    part = min(part, parts);
    return narrow ? (long long)((uint32_t)(total * part) / (uint32_t)parts) : total * part / parts;
  };
  // the request in which place p lies, if it is one of this thread's, and how far in
  auto within = [&](long long p, long long &rest) {
    rest = p - (upto - mine);
    if (rest < 0 || rest >= mine) return -1;
    for (int r = r0;; r++) {
      const long long n = (long long)visible_of(a, clamped_len(a, r)).template steps<WARPS>(s.solo) * items;
      if (rest < n) return r;
      rest -= n;
    }
  };
  int r_lo = a.n_req, r_hi = a.n_req;   // (n_req: the line's end)
  long long in_lo = 0, in_hi = 0;
  const long long lo = cut(first + (s.solo ? warp : 0)), hi = cut(first + (s.solo ? warp : 0) + 1);
  if (few) {
    auto locate = [&](long long p, int &r, long long &in) {
      long long rest;
      const int mine_r = within(p, rest);
      const unsigned who = __ballot_sync(0xffffffffu, mine_r >= 0);
      if (who) {
        r = __shfl_sync(0xffffffffu, mine_r, __ffs(who) - 1);
        in = __shfl_sync(0xffffffffu, rest, __ffs(who) - 1);
      }
    };
    locate(lo, r_lo, in_lo);
    if (whole) locate(hi, r_hi, in_hi);
  } else {
    for (int k = 0; k < (s.solo ? WARPS + 1 : whole ? 2 : 1); k++) {
      long long rest;
      const int r = within(cut(first + k), rest);
      if (r >= 0) { found_r[k] = r; found_into[k] = rest; }
    }
    __syncthreads();
    const int k = s.solo ? warp : 0;
    r_lo = found_r[k]; in_lo = found_into[k];
    if (whole) { r_hi = found_r[k + 1]; in_hi = found_into[k + 1]; }
  }
  long long n = hi - lo;
  if (whole) {   // from the first item that begins at or behind a cut to the first at or behind the next cut
    auto to_item = [&](int r, long long in) {
      if (r >= a.n_req) return 0;
      const int steps = visible_of(a, clamped_len(a, r)).template steps<WARPS>(s.solo), tile = (int)(in % steps);
      return tile ? steps - tile : 0;
    };
    const int skip = to_item(r_lo, in_lo);
    n += to_item(r_hi, in_hi) - skip;
    in_lo += skip;
    if (r_lo < a.n_req && in_lo == (long long)visible_of(a, clamped_len(a, r_lo)).template steps<WARPS>(s.solo) * items) { r_lo++; in_lo = 0; }
  }
  s.r = r_lo;
  s.into = in_lo;
  s.n = (int)n;   // (the host refuses calls that could have more)
  return s;
}

template <typename T, int D, int NT>
struct PaSmem {
  static constexpr int LD = D + 8, HB = 8 * NT, LF = D / 2 + 4;   // (rows of both spread over the banks)
  static constexpr int STAGE = 2 * 16 * LD * 2;                   // bytes: keys and values of a warp's 16
  typedef PaCfg<D, NT> Cfg;
  static constexpr int FO = Cfg::WARPS * 8 * LF;                  // floats in which the warps meet
  static constexpr int BYTES = Cfg::WARPS * Cfg::STAGES * STAGE + (Cfg::TWO ? 2 : 1) * FO * 4;
  static_assert(Cfg::PER_SM * (BYTES + 2500) <= 228 * 1024, "blocks of an SM");
};

template <typename T, int D, int NT>
__global__ void __launch_bounds__(PaCfg<D, NT>::WARPS * 32, PaCfg<D, NT>::PER_SM)
paged_attn_kernel(const __grid_constant__ PagedAttn a) {
  using S = PaSmem<T, D, NT>;
  constexpr int PA_WARPS = PaCfg<D, NT>::WARPS, PA_STAGES = PaCfg<D, NT>::STAGES, PA_THREADS = PA_WARPS * 32;
  constexpr int LD = S::LD, HB = S::HB, LF = S::LF, KD = D / 16;
  extern __shared__ __align__(16) unsigned char pa_smem[];
  __shared__ int4 info[PA_WARPS][PA_STAGES];
  __shared__ float wm[2][PA_WARPS][HB], wl[2][PA_WARPS][HB];   // (two sets: one may still be read while the next is written)
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g4 = lane >> 2, q4 = lane & 3;
  const int items = a.h_kv * a.groups;
  T *const ring = reinterpret_cast<T *>(pa_smem + warp * PA_STAGES * S::STAGE);
  float *const fo0 = reinterpret_cast<float *>(pa_smem + PA_WARPS * PA_STAGES * S::STAGE);   // [warp][8][LF], once or twice
  using Cfg = PaCfg<D, NT>;
  pdl_launch_dependents();

  const Share share = find_share<PA_WARPS>(a, items);
  const int n_steps = share.n;
  const bool solo = share.solo;
  int4 rec = make_int4(-1, 0, 0, 0);
  if (n_steps == 0) {
    if (tid == 0) a.rec[blockIdx.x] = rec;
    return;   // (the whole block, or a warp that no other waits for)
  }

  Cursor<PA_WARPS> load;
  load.solo = solo;
  load.enter(a, share.r, clamped_len(a, share.r));
  {
    const int item = share.into <= INT32_MAX ? (int)share.into / load.steps : (int)(share.into / load.steps);
    load.tile = (int)(share.into - (long long)item * load.steps);
    load.m = item / a.groups;
    load.hg = item - load.m * a.groups;
    load.head_at = load.m * a.head_stride;
  }

  // The next step to be requested: lane (and lane + 16) = row of the warp's 16.  Its table entry is on its way a step ahead of its
  // use.  A row is copied by as many neighbouring lanes as it has pieces of 16 bytes (a row in four pieces of 64 bytes, at fixed
  // offsets from one address per lane, or a bulk copy per row, take fewer instructions and 10 and 30% more time).
  constexpr int VPR = D / 8, COPIES = 16 * VPR / 32;
  int row_page = 0, row_j = 0, row_key = 0;
  bool row_there = false;
  auto look_up = [&]() {
    // (unsigned: of a request of nearly 2^31 tokens the last step ends behind them)
    const uint32_t i = (uint32_t)(solo ? load.tile : load.tile * PA_WARPS + warp) * 16u + (lane & 15);
    row_there = i < (uint32_t)load.v.n;
    row_key = row_there ? load.v.key((int)i) : 0;
    row_j = a.by_size.div(row_key);
    row_page = row_there ? __ldg(load.row + row_j) : 0;
  };
  auto request = [&](int stage) {
    if (row_page < 0 || row_page >= a.n_pages) {
      row_there = false;
      report(a.status, LOCRET_ERR_INVALID);
    }
    const uint32_t mask = __ballot_sync(0xffffffffu, row_there) & 0xffffu;
    const uint32_t at = row_there ? row_page * a.page_stride + (row_key - row_j * a.page_size) * a.token_stride + load.head_at : 0;
    // what the step is, for the warp that will work on it: keys that exist | last of its item, request, item, step of the item
    if (lane == 0) info[warp][stage] = make_int4((int)mask | (load.tile + 1 == load.steps ? 1 << 16 : 0), load.r,
                                                 pack_item(load.m, load.hg), load.tile);
    T *const ks = ring + stage * (S::STAGE / 2), *const vs = ks + 16 * LD;
#pragma unroll
    for (int x = 0; x < COPIES; x++) {
      const int c = x * 32 + lane, row = c / VPR, col = c - row * VPR;
      const uint32_t piece = __shfl_sync(0xffffffffu, at, row) + col;
      const bool ok = mask == 0xffff || (mask >> row & 1);
      cp_async16(ks + row * LD + col * 8, a.k + piece, ok);
      cp_async16(vs + row * LD + col * 8, a.v + piece, ok);
    }
  };
  int to_ask = n_steps;
  look_up();
#pragma unroll
  for (int s = 0; s < PA_STAGES - 1; s++) {
    if (to_ask > 0) {
      request(s);
      load.next(a);
      if (--to_ask > 0) look_up();
    }
    cp_async_commit();
  }

  const int g = a.h / a.h_kv;
  auto load_q = [&](uint32_t (&to)[NT][KD][2], int r, int m, int hg) {
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
      const int head = hg * HB + nt * 8 + g4;   // within the group
      const T *row = static_cast<const T *>(a.q) + r * a.q_req + (m * g + min(head, g - 1)) * a.q_head + q4 * 2;
#pragma unroll
      for (int kk = 0; kk < KD; kk++) {
        to[nt][kk][0] = head < g ? *reinterpret_cast<const uint32_t *>(row + kk * 16) : 0u;
        to[nt][kk][1] = head < g ? *reinterpret_cast<const uint32_t *>(row + kk * 16 + 8) : 0u;
      }
    }
  };
  uint32_t qf[NT][KD][2], qn[NT][KD][2];
  bool first_item = true;
  int set = 0;
  using Weight = PaWeight<T>;
  // Sums, the scale (-inf: no key yet, and at the end of an item without one the output is 0), and what a score may not exceed: NaN
  // before the first keys, which then set a scale whatever their scores are.  It is finite for keys whose scores are all -inf: their
  // softmax is NaN, but beside others they weigh 0.
  float o[NT][KD][4], m_run[NT][2], l_run[NT][2], m_most[NT][2];
  bool fresh = true;                   // the state belongs to no item yet
  int first_tile = 0, stage = 0;
  for (int left = n_steps; left > 0; left--) {
    cp_async_wait<PA_STAGES - 2>();
    __syncwarp();   // the other lanes' copies too; and all lanes are done with the stage that is refilled now
    const int4 step = info[warp][stage];
    if (fresh) {
      fresh = false;
      first_tile = step.w;
      const int m = item_m(step.z), hg = item_hg(step.z);
      // the item's queries, requested when the last one began, and the next one's
      if (first_item) load_q(qn, step.y, m, hg);
      first_item = false;
#pragma unroll
      for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int kk = 0; kk < KD; kk++) { qf[nt][kk][0] = qn[nt][kk][0]; qf[nt][kk][1] = qn[nt][kk][1]; }
      const bool next_head = hg + 1 == a.groups, next_r = next_head && m + 1 == a.h_kv;
      load_q(qn, min(next_r ? step.y + 1 : step.y, a.n_req - 1), next_r ? 0 : next_head ? m + 1 : m, next_head ? 0 : hg + 1);
#pragma unroll
      for (int nt = 0; nt < NT; nt++) {
#pragma unroll
        for (int kk = 0; kk < KD; kk++)
#pragma unroll
          for (int e = 0; e < 4; e++) o[nt][kk][e] = 0.f;
#pragma unroll
        for (int e = 0; e < 2; e++) {
          m_run[nt][e] = -INFINITY;
          m_most[nt][e] = NAN;
          l_run[nt][e] = 0.f;
        }
      }
    }
    if (to_ask > 0) {
      request(stage == 0 ? PA_STAGES - 1 : stage - 1);   // (the stage of the last step)
      load.next(a);
      if (--to_ask > 0) look_up();
    }
    cp_async_commit();

    const T *const ks = ring + stage * (S::STAGE / 2), *const vs = ks + 16 * LD;
    const uint32_t mask = step.x & 0xffff;
    if (mask) {
      float s[NT][4] = {};
#pragma unroll
      for (int kk = 0; kk < KD; kk++) {
        uint32_t a0, a1, a2, a3;
        ldmatrix_x4(a0, a1, a2, a3, ks + (lane & 15) * LD + kk * 16 + (lane >> 4) * 8);
#pragma unroll
        for (int nt = 0; nt < NT; nt++) mma16<T>(s[nt], a0, a1, a2, a3, qf[nt][kk][0], qf[nt][kk][1]);
      }
      // s[nt]: keys g4, g4, g4 + 8, g4 + 8 of heads 2 q4, 2 q4 + 1, 2 q4, 2 q4 + 1
#pragma unroll
      for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int e = 0; e < 4; e++) s[nt][e] *= a.scale_log2;
      if (mask != 0xffff) {
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
          for (int e = 0; e < 4; e++)
            if (!((mask >> (g4 + (e >> 1) * 8)) & 1)) s[nt][e] = -INFINITY;
      }
      bool raise = false;
#pragma unroll
      for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int e = 0; e < 4; e++) raise |= !(s[nt][e] <= m_most[nt][e & 1]);
      if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
          float alpha[2];
#pragma unroll
          for (int e = 0; e < 2; e++) {
            float t = fmaxf(s[nt][e], s[nt][e + 2]);
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, x));
            const float top = fmaxf(fmaxf(m_run[nt][e], -FLT_MAX), t);
            m_most[nt][e] = __fadd_rd(top, Weight::MOST);   // (down: no weight exceeds 2^MOST, however coarse fp32 is at these scores)
            alpha[e] = exp2_fast(m_run[nt][e] - top);
            m_run[nt][e] = top;
            l_run[nt][e] *= alpha[e];
          }
#pragma unroll
          for (int kk = 0; kk < KD; kk++)
#pragma unroll
            for (int e = 0; e < 4; e++) o[nt][kk][e] *= alpha[e & 1];
        }
      }
      // P^T, as the sum of two 16-bit numbers: the high part and what it leaves
      uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int half = 0; half < 2; half++) {
          float p[2];
#pragma unroll
          for (int e = 0; e < 2; e++) {
            p[e] = exp2_fast(s[nt][half * 2 + e] - m_run[nt][e]);
            l_run[nt][e] += p[e];
            p[e] *= Weight::UP;
          }
          const uint32_t hi16 = Half2<T>::pack(p[0], p[1]);
          const float2 back = Half2<T>::unpack(hi16);
          ph[nt][half] = transpose8x8(hi16);
          pl[nt][half] = transpose8x8(Half2<T>::pack(p[0] - back.x, p[1] - back.y));
        }
#pragma unroll
      for (int kk = 0; kk < KD; kk++) {
        uint32_t a0, a1, a2, a3;
        ldmatrix_x4_trans(a0, a1, a2, a3, vs + ((lane & 7) + (lane >> 4) * 8) * LD + kk * 16 + ((lane >> 3) & 1) * 8);
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
          mma16<T>(o[nt][kk], a0, a1, a2, a3, ph[nt][0], ph[nt][1]);
          mma16<T>(o[nt][kk], a0, a1, a2, a3, pl[nt][0], pl[nt][1]);
        }
      }
    }
    __syncwarp();

    const bool ends = step.x >> 16 & 1;
    if (ends && solo) {
      // ---- the warp writes its item, half of the columns at a time through its own part of the buffer
      const int m = item_m(step.z), hg = item_hg(step.z), gh = min(HB, g - hg * HB);
      float *const mine = fo0 + warp * 8 * LF;
#pragma unroll
      for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) l_run[nt][e] += __shfl_xor_sync(0xffffffffu, l_run[nt][e], x);
          if (g4 == 0) { wm[0][warp][nt * 8 + q4 * 2 + e] = m_run[nt][e]; wl[0][warp][nt * 8 + q4 * 2 + e] = l_run[nt][e]; }
        }
#pragma unroll
      for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int side = 0; side < 2; side++) {
#pragma unroll
          for (int kk = 0; kk < KD / 2; kk++)
#pragma unroll
            for (int e = 0; e < 4; e++)
              mine[(q4 * 2 + (e & 1)) * LF + kk * 16 + g4 + (e >> 1) * 8] = o[nt][side * (KD / 2) + kk][e];
          __syncwarp();
#pragma unroll
          for (int x = lane; x < 8 * (D / 8); x += 32) {
            const int hh = x / (D / 8), c = (x - hh * (D / 8)) * 4, head = nt * 8 + hh, col = side * (D / 2) + c;
            if (head >= gh) continue;
            const float top = wm[0][warp][head], l = wl[0][warp][head], inv = top == -INFINITY ? 0.f : 1.0f / (l * PaWeight<T>::UP);
            const float4 f = *reinterpret_cast<const float4 *>(mine + hh * LF + c);
            const int j = m * g + hg * HB + head;
            *reinterpret_cast<uint2 *>(static_cast<T *>(a.out) + step.y * a.out_req + j * a.out_head + col) =
                make_uint2(Half2<T>::pack(f.x * inv, f.y * inv), Half2<T>::pack(f.z * inv, f.w * inv));
            if (a.lse && col == 0)
              a.lse[(size_t)step.y * a.h + j] = top == -INFINITY ? top : (top + log2f(l)) * 0.6931471805599453f;
          }
          __syncwarp();
        }
      fresh = true;
    } else if (ends || left == 1) {
      // ---- the warps meet: each leaves its sums as they are, and who adds them up weighs them by their scales
      const bool whole = ends && first_tile == 0, begins = first_tile == 0;
      const int m = item_m(step.z), hg = item_hg(step.z), gh = min(HB, g - hg * HB);
#pragma unroll
      for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int e = 0; e < 2; e++) {
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) l_run[nt][e] += __shfl_xor_sync(0xffffffffu, l_run[nt][e], x);
          if (g4 == 0) { wm[set][warp][nt * 8 + q4 * 2 + e] = m_run[nt][e]; wl[set][warp][nt * 8 + q4 * 2 + e] = l_run[nt][e]; }
        }
      float *const part = a.part + ((size_t)blockIdx.x * 2 + (begins ? 1 : 0)) * (HB * (D + 2));
#pragma unroll
      for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int side = 0; side < 2; side++) {
          // two buffers: of a side's, every read was done before the barrier of the other; one: wait for the reads
          if (!Cfg::TWO) __syncthreads();
          float *const fo = fo0 + (Cfg::TWO ? side * S::FO : 0);
#pragma unroll
          for (int kk = 0; kk < KD / 2; kk++)
#pragma unroll
            for (int e = 0; e < 4; e++)
              fo[(warp * 8 + q4 * 2 + (e & 1)) * LF + kk * 16 + g4 + (e >> 1) * 8] = o[nt][side * (KD / 2) + kk][e];
          __syncthreads();
          for (int x = tid; x < 8 * (D / 8); x += PA_THREADS) {   // (head, four columns of this half)
            const int hh = x / (D / 8), c = (x - hh * (D / 8)) * 4, head = nt * 8 + hh, col = side * (D / 2) + c;
            if (head >= gh) continue;
            float top = wm[set][0][head], l = 0.f;
#pragma unroll
            for (int v = 1; v < PA_WARPS; v++) top = fmaxf(top, wm[set][v][head]);
            const float ref = top == -INFINITY ? 0.f : top;
            float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int v = 0; v < PA_WARPS; v++) {
              const float w = exp2_fast(wm[set][v][head] - ref);
              const float4 f = *reinterpret_cast<const float4 *>(fo + (v * 8 + hh) * LF + c);
              sum.x = fmaf(w, f.x, sum.x); sum.y = fmaf(w, f.y, sum.y); sum.z = fmaf(w, f.z, sum.z); sum.w = fmaf(w, f.w, sum.w);
              l = fmaf(w, wl[set][v][head], l);
            }
            const int j = m * g + hg * HB + head;
            if (whole) {
              const float inv = top == -INFINITY ? 0.f : 1.0f / (l * PaWeight<T>::UP);
              *reinterpret_cast<uint2 *>(static_cast<T *>(a.out) + step.y * a.out_req + j * a.out_head + col) =
                  make_uint2(Half2<T>::pack(sum.x * inv, sum.y * inv), Half2<T>::pack(sum.z * inv, sum.w * inv));
              if (a.lse && col == 0) a.lse[(size_t)step.y * a.h + j] = top == -INFINITY ? top : (top + log2f(l)) * 0.6931471805599453f;
            } else {
              *reinterpret_cast<float4 *>(part + head * D + col) = sum;
              if (col == 0) *reinterpret_cast<float2 *>(part + HB * D + head * 2) = make_float2(top, l);
            }
          }
        }
      set ^= 1;
      if (!whole) {
        if (begins) { rec.x = step.y; rec.y = step.z; }
        else rec.z = ends ? 2 : 1;
      }
      fresh = true;
    }
    stage = stage + 1 == PA_STAGES ? 0 : stage + 1;
  }
  cp_async_wait<0>();
  if (tid == 0) a.rec[blockIdx.x] = rec;
}

// Block (b, head) joins that head of the item that begins in block b's part of the line and ends in another's.  A chain of
// latencies (records, then parts): a warp's lanes take four columns each, and JOIN_WARPS * JOIN_BATCH parts are requested before
// one is used (one request of 6000 tokens, 38 parts an item: 23 us with a warp per head and a part after the other, 4.8 now).  Most
// blocks find nothing to join and end: small ones, so that all of them fit at once (four warps: 61 requests 1.2 us longer).
constexpr int JOIN_WARPS = 2, JOIN_BATCH = 10;

template <typename T, int D, int NT>
__global__ void __launch_bounds__(JOIN_WARPS * 32) paged_join_kernel(const __grid_constant__ PagedAttn a) {
  constexpr int HB = 8 * NT, PART = HB * (D + 2);
  __shared__ float4 sums[JOIN_WARPS][D / 4];
  __shared__ float ls[JOIN_WARPS];
  const int b = blockIdx.x, head = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  pdl_wait();
  // its parts: the second of block b, the first of the blocks behind it up to the one where it ends
  int4 rec = make_int4(0, 0, 2, 0);
  if (b + lane < gridDim.x) rec = __ldcg(a.rec + b + lane);
  const int r = __shfl_sync(0xffffffffu, rec.x, 0), item = __shfl_sync(0xffffffffu, rec.y, 0);
  if (r < 0) return;
  const int g = a.h / a.h_kv, m = item_m(item), hg = item_hg(item);
  if (head >= g - hg * HB) return;
  int n = 1;
  for (int at = b;; at += 32) {
    if (at > b) rec.z = at + lane < gridDim.x ? __ldcg(&a.rec[at + lane].z) : 2;
    const unsigned ends = __ballot_sync(0xffffffffu, rec.z == 2 && at + lane > b);
    if (ends) { n = at - b + __ffs(ends); break; }
  }
  const float *const first = a.part + ((size_t)b * 2 + 1) * PART, *const others = a.part + (size_t)b * 2 * PART;   // (part i > 0)
  auto part = [&](int i) { return i == 0 ? first : others + (size_t)i * 2 * PART; };
  float4 o[JOIN_BATCH];
  float2 ml[JOIN_BATCH];
  auto fetch = [&](int i0) {
#pragma unroll
    for (int u = 0; u < JOIN_BATCH; u++) {
      const int i = i0 + u * JOIN_WARPS + warp;
      o[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      ml[u] = make_float2(-INFINITY, 0.f);
      if (i < n) ml[u] = __ldcg(reinterpret_cast<const float2 *>(part(i) + HB * D) + head);
      if (i < n && lane < D / 4) o[u] = __ldcg(reinterpret_cast<const float4 *>(part(i) + head * D) + lane);
    }
  };
  fetch(0);
  float top = -INFINITY;
  for (int i = lane; i < n; i += 32) top = fmaxf(top, __ldcg(part(i) + HB * D + head * 2));
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
  const float ref = top == -INFINITY ? 0.f : top;
  float l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = 0;;) {
#pragma unroll
    for (int u = 0; u < JOIN_BATCH; u++) {
      const float w = exp2f(ml[u].x - ref);
      acc.x = fmaf(w, o[u].x, acc.x); acc.y = fmaf(w, o[u].y, acc.y);
      acc.z = fmaf(w, o[u].z, acc.z); acc.w = fmaf(w, o[u].w, acc.w);
      l = fmaf(w, ml[u].y, l);
    }
    i0 += JOIN_BATCH * JOIN_WARPS;
    if (i0 >= n) break;
    fetch(i0);
  }
  if (lane < D / 4) sums[warp][lane] = acc;
  if (lane == 0) ls[warp] = l;
  __syncthreads();
  if (warp > 0 || lane >= D / 4) return;
#pragma unroll
  for (int s = 1; s < JOIN_WARPS; s++) {
    const float4 x = sums[s][lane];
    acc.x += x.x; acc.y += x.y; acc.z += x.z; acc.w += x.w;
    l += ls[s];
  }
  const int j = m * g + hg * HB + head;
  const float inv = top == -INFINITY ? 0.f : 1.0f / (l * PaWeight<T>::UP);   // (no part has seen a key)
  *reinterpret_cast<uint2 *>(static_cast<T *>(a.out) + r * a.out_req + j * a.out_head + lane * 4) =
      make_uint2(Half2<T>::pack(acc.x * inv, acc.y * inv), Half2<T>::pack(acc.z * inv, acc.w * inv));
  if (a.lse && lane == 0) a.lse[(size_t)r * a.h + j] = top == -INFINITY ? top : (top + log2f(l)) * 0.6931471805599453f;
}

int heads_per_block(int h, int h_kv) { return h / h_kv > 8 ? 16 : 8; }
int paged_blocks() { return sm_count_of_current_device() * 2; }
static_assert(PaCfg<64, 1>::PER_SM == 2 && PaCfg<96, 1>::PER_SM == 2 && PaCfg<128, 1>::PER_SM == 2 && PaCfg<128, 2>::PER_SM == 2, "the grid");
size_t part_floats(int h, int h_kv, int d) { return (size_t)heads_per_block(h, h_kv) * (d + 2); }

template <typename T, int D, int NT>
cudaError_t launch(PagedAttn &a, long long most_keys, cudaStream_t st) {
  using S = PaSmem<T, D, NT>;
  static PerDeviceFlag flag;
  cudaError_t e = allow_dynamic_smem(paged_attn_kernel<T, D, NT>, S::BYTES, flag);
  if (e != cudaSuccess) return e;
  const int blocks = paged_blocks(), g = a.h / a.h_kv;
  // Where no request can be longer than a few steps, blocks take whole items and there is no second launch - if there are items
  // for half of the blocks, or hardly a step to divide (eight KV heads of 128, 20 requests of up to 400 tokens: 14.5 us divided,
  // 13.1 whole; 32 of 96, eight of 300: 12.9, 10.2; but one request of 400: 8.1, 11.3).
  const long long most_steps = (most_keys + S::Cfg::WARPS * 16 - 1) / (S::Cfg::WARPS * 16);
  a.whole = most_steps <= 2 || (most_steps <= PA_WHOLE && 2ll * a.n_req * a.h_kv * a.groups >= blocks);
  e = launch_kernel(paged_attn_kernel<T, D, NT>, dim3(blocks), dim3(S::Cfg::WARPS * 32), S::BYTES, st, false, a);
  if (e != cudaSuccess || a.whole) return e;
  return launch_kernel(paged_join_kernel<T, D, NT>, dim3(blocks, g < 8 * NT ? g : 8 * NT), dim3(JOIN_WARPS * 32), 0, st, true, a);
}

template <typename T>
cudaError_t launch_by_size(PagedAttn &a, int d, int nt, long long most_keys, cudaStream_t st) {
  if (nt == 1) return d == 64 ? launch<T, 64, 1>(a, most_keys, st) : d == 96 ? launch<T, 96, 1>(a, most_keys, st) : launch<T, 128, 1>(a, most_keys, st);
  return d == 64 ? launch<T, 64, 2>(a, most_keys, st) : d == 96 ? launch<T, 96, 2>(a, most_keys, st) : launch<T, 128, 2>(a, most_keys, st);
}

bool heads_ok(int32_t h, int32_t h_kv, int32_t d) {
  return h >= 1 && h_kv >= 1 && h <= 65536 && h % h_kv == 0 && (d == 64 || d == 96 || d == 128);
}
bool aligned16p(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace
}  // namespace locret

using namespace locret;

extern "C" int locret_paged_attention_workspace(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int64_t *bytes) {
  if (!bytes || !heads_ok(n_q_heads, n_kv_heads, head_dim)) return LOCRET_ERR_INVALID;
  *bytes = (int64_t)paged_blocks() * (sizeof(int4) + 2 * sizeof(float) * part_floats(n_q_heads, n_kv_heads, head_dim));
  return LOCRET_OK;
}

extern "C" int locret_paged_attention(const void *q, int64_t q_req, int64_t q_head, const locret_pages *pages,
                                      const int32_t *table, int64_t table_stride, int32_t width, const int32_t *lens,
                                      int32_t n_req, int32_t n_q_heads, float scale, int32_t window, int32_t sinks, void *out,
                                      int64_t out_req, int64_t out_head, float *lse, int32_t *status, void *workspace,
                                      int64_t workspace_bytes, void *stream) {
  if (!pages || !pages_ok(*pages) || !heads_ok(n_q_heads, pages->n_kv_heads, pages->head_dim)) return LOCRET_ERR_INVALID;
  const float scale_log2 = scale * 1.4426950408889634f;   // (infinite, it would make NaN of a score of 0)
  if (n_req < 0 || n_req > LOCRET_MAX_REQUESTS || width < 1 || table_stride < 0 || (n_req > 1 && table_stride < width) ||
      window < 0 || sinks < 0 || !isfinite(scale_log2))
    return LOCRET_ERR_INVALID;
  if ((q_req | q_head | out_req | out_head) & 7 || !aligned16p(q) || !aligned16p(out) || !aligned16p(workspace)) return LOCRET_ERR_INVALID;
  const long double span = (long double)(pages->n_pages - 1) * pages->page_stride + (long double)(pages->page_size - 1) * pages->token_stride +
                           (long double)(pages->n_kv_heads - 1) * pages->head_stride + pages->head_dim;
  if (span / 8 >= 4294967296.0L) return LOCRET_ERR_INVALID;
  // steps of the longest line there could be, a block's share of it (2^31 steps would take a block ten minutes)
  const long double steps = ((long double)width * pages->page_size / 64 + 1) * n_req * n_q_heads;
  if (steps / paged_blocks() >= 2147483648.0L) return LOCRET_ERR_INVALID;
  if (n_req == 0) return LOCRET_OK;
  if (!q || !table || !lens || !out || !workspace) return LOCRET_ERR_INVALID;
  int64_t need = 0;
  locret_paged_attention_workspace(n_q_heads, pages->n_kv_heads, pages->head_dim, &need);
  if (workspace_bytes < need) return LOCRET_ERR_CAPACITY;
  const int hb = heads_per_block(n_q_heads, pages->n_kv_heads), g = n_q_heads / pages->n_kv_heads;
  PagedAttn a = {};
  a.q = q; a.out = out; a.lse = lse; a.status = status;
  a.rec = static_cast<int4 *>(workspace);
  a.part = reinterpret_cast<float *>(a.rec + paged_blocks());
  a.table = table; a.lens = lens; a.table_stride = table_stride;
  a.k = static_cast<const uint4 *>(pages->k); a.v = static_cast<const uint4 *>(pages->v);
  a.page_stride = (uint32_t)(pages->page_stride / 8); a.head_stride = (uint32_t)(pages->head_stride / 8);
  a.token_stride = (uint32_t)(pages->token_stride / 8);
  a.n_pages = pages->n_pages; a.page_size = pages->page_size; a.by_size = FastDiv(pages->page_size);
  a.q_req = q_req; a.q_head = q_head; a.out_req = out_req; a.out_head = out_head;
  a.width = width; a.n_req = n_req; a.h = n_q_heads; a.h_kv = pages->n_kv_heads; a.groups = (g + hb - 1) / hb;
  a.window = window; a.sinks = sinks;
  a.scale_log2 = scale_log2;
  long long most_keys = (long long)width * pages->page_size;
  if (window > 0 && (long long)window + sinks < most_keys) most_keys = (long long)window + sinks;
  const cudaError_t e = pages->dtype == LOCRET_BF16 ? launch_by_size<bf16>(a, pages->head_dim, hb / 8, most_keys, (cudaStream_t)stream)
                                                    : launch_by_size<__half>(a, pages->head_dim, hb / 8, most_keys, (cudaStream_t)stream);
  if (e != cudaSuccess) { cudaGetLastError(); return LOCRET_ERR_CUDA; }
  return LOCRET_OK;
}
