// A pool of pages shared by several requests: the bookkeeping of a step, and a layer's retained units into pages.
#include "../../include/locret.h"
#include "common.cuh"
#include "paged.cuh"

namespace locret {
namespace {

// ---------------------------------------------------------------- one step's bookkeeping
// Four prefix sums over the requests decide everything: rows of the step, pages given back, pages needed, and through the
// last two which entry of the free list is whose.  Nothing here is bound by bytes (a busy server's step moves 130 KB): it is a
// chain of latencies (lengths -> sums -> entries -> slots), so one launch does all of it.  Every block of a cluster computes
// the sums for itself (at most LOCRET_MAX_REQUESTS lengths from L2), and the blocks share the entries and rows.  The one
// barrier of the cluster stands between reading and writing: behind it lens_out and n_free_out may overwrite their inputs, and
// pages that were pushed onto the list can be taken from it.
constexpr int PS_THREADS = 512, PS_WARPS = PS_THREADS / 32, PS_SHARE = 8;
constexpr int PS_PER = LOCRET_MAX_REQUESTS / PS_THREADS;   // requests of a thread, at most

struct PagesStepArgs {
  int32_t *table;
  long long table_stride;
  const int32_t *lens_in, *new_lens, *n_free_in;
  int32_t *lens_out, *free_pages, *n_free_out, *positions, *starts, *status;
  int64_t *slots;
  int width, n_req, page_size, capacity, n_tok, vec;   // vec: slots and positions are aligned for 16-byte stores
  FastDiv by_page;
};

// Exclusive prefix sums over the block's threads of two 64-bit numbers each; sum0, sum1 are the whole sums.
__device__ void block_scan(long long &v0, long long &v1, long long &sum0, long long &sum1, longlong2 *warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  auto warp_scan = [&](long long v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += y;
    }
    return v;
  };
  const long long x0 = warp_scan(v0), x1 = warp_scan(v1);
  if (lane == 31) warp_sums[warp] = make_longlong2(x0, x1);
  __syncthreads();
  const longlong2 mine = lane < warps ? warp_sums[lane] : make_longlong2(0, 0);
  const long long w0 = warp_scan(mine.x), w1 = warp_scan(mine.y);
  sum0 = __shfl_sync(0xffffffffu, w0, 31);
  sum1 = __shfl_sync(0xffffffffu, w1, 31);
  v0 = x0 - v0 + (warp ? __shfl_sync(0xffffffffu, w0, warp - 1) : 0);
  v1 = x1 - v1 + (warp ? __shfl_sync(0xffffffffu, w1, warp - 1) : 0);
}

// The request whose range [first[r], first[r + 1]) holds i, 0 <= i, i < first[n] (which is not read).
__device__ __forceinline__ int owner(const int *first, int n, int i) {
  int lo = 0, hi = n;   // first[lo] <= i < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= i) lo = mid; else hi = mid;
  }
  return lo;
}

constexpr int REFUSED = INT32_MIN;   // in place of a request's length

// A thread's requests are its `per` ones from r0 on.  CLUSTER: several blocks (else the one needs no more than its own barriers).
template <bool CLUSTER>
__global__ void __launch_bounds__(PS_THREADS) pages_step_kernel(const __grid_constant__ PagesStepArgs a) {
  extern __shared__ int ps_smem[];
  int *const starts = ps_smem, *const need0 = starts + a.n_req + 1, *const len = need0 + a.n_req + 1;
  __shared__ longlong2 sums_a[PS_WARPS], sums_b[PS_WARPS];
  __shared__ int taken;
  const int tid = threadIdx.x, lane = tid & 31, threads = blockDim.x, rank = CLUSTER ? blockIdx.x : 0, n_blocks = CLUSTER ? gridDim.x : 1;
  const int per = (a.n_req + threads - 1) / threads;   // <= PS_PER
  const int r0 = min(a.n_req, tid * per), mine = min(a.n_req, r0 + per) - r0;
  const int page = a.page_size;
  const long long room = min((long long)a.width * page, (long long)INT32_MAX);
  auto pages_of = [&](int n) { return n ? a.by_page.div(n - 1) + 1 : 0; };
  if (tid == 0) taken = 0;

  // lengths before (REFUSED where they are none) and numbers of new tokens; rows of every request; pages that come back
  int n_free = *a.n_free_in, n[PS_PER], x[PS_PER];
#pragma unroll
  for (int i = 0; i < PS_PER; i++) {
    n[i] = i < mine ? a.lens_in[r0 + i] : 0;
    x[i] = i < mine ? a.new_lens[r0 + i] : 0;
  }
  long long row = 0, push = 0, total_rows, total_back;
#pragma unroll
  for (int i = 0; i < PS_PER; i++) {
    if (i >= per) break;   // (here and below: the same for every thread)
    if (n[i] < 0 || n[i] > room) n[i] = REFUSED;
    row += max(x[i], 0);
    if (x[i] < 0 && n[i] != REFUSED) push += pages_of(n[i]);
  }
  const bool bad_list = n_free < 0 || n_free > a.capacity;
  n_free = min(max(n_free, 0), a.capacity);
  block_scan(row, push, total_rows, total_back, sums_a);
  const bool too_many = n_free + total_back > a.capacity;   // (some page is on the list twice)
  const int top = (int)min(n_free + total_back, (long long)a.capacity);

  // who is refused before the list is looked at; pages the others need
  long long want = 0, none = 0, total_need, total_none;
  int code = 0, more[PS_PER], back[PS_PER];
#pragma unroll
  for (int i = 0; i < PS_PER; i++) {
    if (i >= per) break;
    more[i] = 0;
    back[i] = x[i] < 0 && n[i] != REFUSED ? pages_of(n[i]) : 0;
    if (i < mine) starts[r0 + i] = (int)min(row, (long long)INT32_MAX);
    if (n[i] == REFUSED) {
      code = min(code, LOCRET_ERR_INVALID);
    } else if (x[i] > 0) {
      if ((long long)n[i] + x[i] > room || row + x[i] > a.n_tok) {
        n[i] = REFUSED;
        code = min(code, LOCRET_ERR_CAPACITY);
      } else {
        more[i] = pages_of(n[i] + x[i]) - pages_of(n[i]);
        want += more[i];
      }
    }
    row += max(x[i], 0);
  }
  block_scan(want, none, total_need, total_none, sums_b);
  int last = 0;   // pages taken: the requests that get theirs come before the first that does not
#pragma unroll
  for (int i = 0; i < PS_PER; i++) {
    if (i >= per) break;
    int first = (int)min(want, (long long)top);
    want += more[i];
    if (more[i] > 0) {
      if (want > top) {   // (and so is every later request that needs a page)
        n[i] = REFUSED;
        first = top;
        code = min(code, LOCRET_ERR_CAPACITY);
      } else {
        last = (int)want;
      }
    }
    if (i < mine) { need0[r0 + i] = first; len[r0 + i] = n[i]; }
  }
  last = __reduce_max_sync(0xffffffffu, last);
  if (lane == 0 && last) atomicMax(&taken, last);
  if (tid == 0) {
    starts[a.n_req] = (int)min(total_rows, (long long)INT32_MAX);
    if (bad_list || too_many) code = min(code, LOCRET_ERR_INVALID);
  }
  if (code && rank == 0) report(a.status, code);

  // ended requests: their pages onto the list, one warp for each request, over all blocks
  if (total_back) {
#pragma unroll
    for (int i = 0; i < PS_PER; i++) {
      if (i >= per) break;
      const int at = (int)min(push, (long long)INT32_MAX);
      push += back[i];
      for (unsigned todo = __ballot_sync(0xffffffffu, back[i] > 0); todo; todo &= todo - 1) {
        const int src = __ffs(todo) - 1;
        const int c = __shfl_sync(0xffffffffu, back[i], src), first = __shfl_sync(0xffffffffu, at, src),
                  rr = __shfl_sync(0xffffffffu, r0 + i, src);
        const int32_t *from = a.table + rr * a.table_stride;
        for (int j0 = rank * 32 + lane; j0 < c; j0 += 4 * n_blocks * 32) {   // (four at a time on their way)
          int32_t p[4];
#pragma unroll
          for (int u = 0; u < 4; u++) p[u] = j0 + u * n_blocks * 32 < c ? from[j0 + u * n_blocks * 32] : 0;
#pragma unroll
          for (int u = 0; u < 4; u++) {
            const int j = j0 + u * n_blocks * 32;
            const long long to = (long long)n_free + first + j;
            if (j < c && to < a.capacity) a.free_pages[to] = p[u];
          }
        }
      }
    }
  }

  // everything that is read has been read, and what was pushed can be seen
  if (CLUSTER) asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  else __syncthreads();

  const int n_taken = taken;   // (need0 of a request behind the last that takes pages is no less)
  for (int r = rank * threads + tid; r < a.n_req; r += n_blocks * threads) {
    const int x = a.new_lens[r], n = len[r];
    a.starts[r] = starts[r];
    if (n == REFUSED) {
      if (a.lens_out != a.lens_in) a.lens_out[r] = a.lens_in[r];
    } else {
      a.lens_out[r] = x < 0 ? 0 : n + x;
    }
  }
  if (rank == 0 && tid == 0) {
    a.starts[a.n_req] = starts[a.n_req];
    *a.n_free_out = top - n_taken;
  }
  // the table's new entries
  for (int k = rank * threads + tid; k < n_taken; k += n_blocks * threads) {
    const int r = owner(need0, a.n_req, k);
    a.table[r * a.table_stride + pages_of(len[r]) + k - need0[r]] = a.free_pages[top - 1 - k];
  }
  // the rows, four in a row for each thread (one search)
  const int n_rows = starts[a.n_req];
  for (long long t0 = 4ll * (rank * threads + tid); t0 < a.n_tok; t0 += 4ll * n_blocks * threads) {
    const int count = (int)min(4ll, a.n_tok - t0);
    int64_t slot[4];
    int pos[4], p[4], off[4], r = t0 < n_rows ? owner(starts, a.n_req, (int)t0) : 0;
    // four rows of one request (a prompt's), in two pages at most, or whatever they are
    const int p0 = count == 4 && page >= 4 && t0 + 4 <= n_rows && starts[r + 1] >= (int)t0 + 4 && len[r] != REFUSED
                       ? len[r] + ((int)t0 - starts[r]) : -1;
    if (p0 >= 0) {
      const int old = pages_of(len[r]), j0 = a.by_page.div(p0), o0 = p0 - j0 * page, j1 = o0 + 4 > page ? j0 + 1 : j0;
      const int32_t *const row = a.table + r * a.table_stride;
      const int32_t *const fresh = a.free_pages + (top - 1 - need0[r] + old);   // (page j of the request: fresh[-j])
      const int a0 = *(j0 < old ? row + j0 : fresh - j0), a1 = *(j1 < old ? row + j1 : fresh - j1);
      const bool ok0 = a0 >= 0 && a0 < a.capacity, ok1 = a1 >= 0 && a1 < a.capacity;
      if (!ok0 || !ok1) report(a.status, LOCRET_ERR_INVALID);
      const int64_t at0 = (int64_t)a0 * page + o0, at1 = (int64_t)a1 * page + o0 - page;
#pragma unroll
      for (int u = 0; u < 4; u++) {
        pos[u] = p0 + u;
        p[u] = off[u] = 0;
        slot[u] = o0 + u < page ? (ok0 ? at0 + u : -1) : (ok1 ? at1 + u : -1);
      }
    } else
#pragma unroll
    for (int u = 0; u < 4; u++) {
      const int t = (int)t0 + u;
      slot[u] = -1;
      pos[u] = p[u] = off[u] = 0;
      if (u < count && t < n_rows) {
        while (starts[r + 1] <= t) r++;   // (ends: t < n_rows = starts[n_req])
        const int n = len[r], i = t - starts[r];
        if (n != REFUSED) {
          pos[u] = n + i;
          const int j = a.by_page.div(pos[u]), old = pages_of(n);
          off[u] = pos[u] - j * page;
          p[u] = j < old ? a.table[r * a.table_stride + j] : a.free_pages[top - 1 - (need0[r] + j - old)];
          slot[u] = -2;   // (found, and to be made of p and off)
        } else {
          pos[u] = (int)max(0LL, min((long long)a.lens_in[r] + i, (long long)INT32_MAX));
        }
      }
    }
#pragma unroll
    for (int u = 0; u < 4; u++)
      if (slot[u] == -2) {
        if (p[u] >= 0 && p[u] < a.capacity) slot[u] = (int64_t)p[u] * page + off[u];
        else { slot[u] = -1; report(a.status, LOCRET_ERR_INVALID); }
      }
    if (count == 4 && a.vec) {
      reinterpret_cast<longlong2 *>(a.slots + t0)[0] = make_longlong2(slot[0], slot[1]);
      reinterpret_cast<longlong2 *>(a.slots + t0)[1] = make_longlong2(slot[2], slot[3]);
      *reinterpret_cast<int4 *>(a.positions + t0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
    } else {
#pragma unroll
      for (int u = 0; u < 4; u++)
        if (u < count) { a.slots[t0 + u] = slot[u]; a.positions[t0 + u] = pos[u]; }
    }
  }
}

// ---------------------------------------------------------------- a layer's units into pages
// Bound by memory: 2 x 2 d bytes read and written per unit.  One 16-byte piece of a key and of a value per thread.
__global__ void __launch_bounds__(256)
export_pages_kernel(const bf16 *__restrict__ k_rot, const bf16 *__restrict__ v, const int32_t *__restrict__ rank, int cap, int d,
                    int len, int ranked_len, const int32_t *__restrict__ table, PageView pg, int32_t *status) {
  const int per_row = d / 8, m = blockIdx.y;
  const long long x = (long long)blockIdx.x * 256 + threadIdx.x;
  if (x >= (long long)len * per_row) return;
  const int i = (int)(x / per_row), c = ((int)(x - (long long)i * per_row)) * 8;
  const int pos = i < ranked_len ? rank[(size_t)m * cap + i] : i;
  const int j = pg.by_size.div(pos), p = pos >= 0 && pos < len ? table[j] : -1;
  if (p < 0 || p >= pg.n_pages) { report(status, LOCRET_ERR_INVALID); return; }
  const size_t src = ((size_t)m * cap + i) * d + c;
  const long long dst = p * pg.page_stride + m * pg.head_stride + (pos - j * pg.page_size) * pg.token_stride + c;
  *reinterpret_cast<uint4 *>(static_cast<bf16 *>(pg.k) + dst) = *reinterpret_cast<const uint4 *>(k_rot + src);
  *reinterpret_cast<uint4 *>(static_cast<bf16 *>(pg.v) + dst) = *reinterpret_cast<const uint4 *>(v + src);
}

}  // namespace

cudaError_t launch_export_pages(const bf16 *k_rot, const bf16 *v, const int32_t *rank, int h_kv, int d, int cap, int len,
                                int ranked_len, const int32_t *table, const locret_pages &pages, int32_t *status, cudaStream_t st) {
  const long long threads = (long long)len * (d / 8);
  export_pages_kernel<<<dim3((unsigned)((threads + 255) / 256), h_kv), 256, 0, st>>>(k_rot, v, rank, cap, d, len, ranked_len,
                                                                                    table, page_view(pages), status);
  return cudaGetLastError();
}

}  // namespace locret

using namespace locret;

// Blocks of the widest cluster of pages_step_kernel on the current device (0: an error), found out once for each.
static int max_cluster() {
  static int found[MAX_DEVICES] = {};
  int dev = 0;
  if (current_device_index(&dev) != cudaSuccess) { cudaGetLastError(); return 0; }
  if (found[dev]) return found[dev];
  constexpr int smem = sizeof(int) * (3 * LOCRET_MAX_REQUESTS + 2);
  if (cudaFuncSetAttribute(pages_step_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  int blocks = 8, clusters = 0;
  if (cudaFuncSetAttribute(pages_step_kernel<true>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(16);
    cfg.blockDim = dim3(PS_THREADS);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 16;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&clusters, pages_step_kernel<true>, &cfg) == cudaSuccess && clusters > 0) blocks = 16;
  }
  cudaGetLastError();
  return found[dev] = blocks;
}

extern "C" int locret_pages_step(int32_t *table, int64_t table_stride, int32_t width, const int32_t *lens_in, int32_t *lens_out,
                                 const int32_t *new_lens, int32_t n_req, int32_t page_size, int32_t *free_pages,
                                 int32_t capacity, const int32_t *n_free_in, int32_t *n_free_out, int32_t n_tok, int64_t *slots,
                                 int32_t *positions, int32_t *starts, int32_t *status, void *stream) {
  if (n_req < 0 || n_req > LOCRET_MAX_REQUESTS || n_tok < 0 || page_size < 1 || width < 1 || capacity < 1 || table_stride < 0)
    return LOCRET_ERR_INVALID;
  if (!free_pages || !n_free_in || !n_free_out || !starts || (n_tok && (!slots || !positions))) return LOCRET_ERR_INVALID;
  if (n_req && (!table || !lens_in || !lens_out || !new_lens || (n_req > 1 && table_stride < width))) return LOCRET_ERR_INVALID;
  const int vec = ((reinterpret_cast<uintptr_t>(slots) | reinterpret_cast<uintptr_t>(positions)) & 15u) == 0;
  const PagesStepArgs a = {table, table_stride, lens_in, new_lens, n_free_in, lens_out, free_pages, n_free_out, positions,
                           starts, status, slots, width, n_req, page_size, capacity, n_tok, vec, FastDiv(page_size)};
  // One block where a thread has no more than an eighth of a request and four rows to do, and no wider than that needs; else a
  // cluster, of sixteen blocks where the device takes that many (2000 requests, 77 thousand rows: 18.8 us with eight, 15.3 with
  // sixteen).
  const int per_thread = n_tok / 4 > PS_SHARE * n_req ? n_tok / 4 + 1 : PS_SHARE * n_req;
  const int most = max_cluster();
  if (most == 0) return LOCRET_ERR_CUDA;
  int threads = 128, blocks = 1;
  while (threads < PS_THREADS && threads < per_thread) threads *= 2;
  while (blocks < most && blocks * threads < per_thread) blocks *= 2;
  const size_t smem = sizeof(int) * (3 * (size_t)n_req + 2);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = (cudaStream_t)stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = blocks;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = blocks > 1 ? 1 : 0;
  if (cudaLaunchKernelEx(&cfg, blocks > 1 ? pages_step_kernel<true> : pages_step_kernel<false>, a) != cudaSuccess) {
    cudaGetLastError();
    return LOCRET_ERR_CUDA;
  }
  return LOCRET_OK;
}
