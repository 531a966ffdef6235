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
constexpr int PS_THREADS = 512, PS_WARPS = PS_THREADS / 32, PS_MAX_BLOCKS = 8;

struct PagesStepArgs {
  int32_t *table;
  long long table_stride;
  const int32_t *lens_in, *new_lens, *n_free_in;
  int32_t *lens_out, *free_pages, *n_free_out, *positions, *starts, *status;
  int64_t *slots;
  int width, n_req, page_size, capacity, n_tok;
};

// Exclusive prefix sum over the block's threads of one 64-bit number each; *total is the whole sum.
__device__ long long block_scan(long long v, long long *warp_sums, long long *total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();   // (the last call's readers of warp_sums are done)
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  long long before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < PS_WARPS; w++) {
    const long long s = warp_sums[w];
    if (w < warp) before += s;
    sum += s;
  }
  *total = sum;
  return before + x - v;
}

// The request whose range [first[r], first[r + 1]) holds i; 0 <= i < first[n].
__device__ __forceinline__ int owner(const int *first, int n, int i) {
  int lo = 0, hi = n;   // first[lo] <= i < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= i) lo = mid; else hi = mid;
  }
  return lo;
}

constexpr int REFUSED = INT32_MIN;   // in place of a request's length

__global__ void __launch_bounds__(PS_THREADS) pages_step_kernel(const __grid_constant__ PagesStepArgs a) {
  extern __shared__ int ps_smem[];
  int *const starts = ps_smem, *const need0 = starts + a.n_req + 1, *const len = need0 + a.n_req + 1;
  __shared__ long long warp_sums[PS_WARPS];
  const int tid = threadIdx.x, rank = blockIdx.x, n_blocks = gridDim.x;
  const int per = (a.n_req + PS_THREADS - 1) / PS_THREADS;
  const int r0 = min(a.n_req, tid * per), r1 = min(a.n_req, r0 + per);
  const int page = a.page_size;
  const long long room = min((long long)a.width * page, (long long)INT32_MAX);
  auto pages_of = [&](long long n) { return (int)((n + page - 1) / page); };   // (n <= room: fits)

  // rows of every request; pages that come back
  long long rows = 0, back = 0, total_rows, total_back, total_need;
  for (int r = r0; r < r1; r++) {
    const int n = a.lens_in[r], x = a.new_lens[r];
    const bool bad = n < 0 || n > room;
    rows += max(x, 0);
    if (x < 0 && !bad) back += pages_of(n);
    len[r] = bad ? REFUSED : n;
  }
  int n_free = *a.n_free_in;
  const bool bad_list = n_free < 0 || n_free > a.capacity;
  n_free = min(max(n_free, 0), a.capacity);
  long long row = block_scan(rows, warp_sums, &total_rows);
  long long push = block_scan(back, warp_sums, &total_back);
  const bool too_many = n_free + total_back > a.capacity;   // (some page is on the list twice)
  const int top = (int)min(n_free + total_back, (long long)a.capacity);

  // who is refused before the list is looked at; pages the others need
  long long need = 0;
  int code = 0;
  for (int r = r0; r < r1; r++) {
    const int x = a.new_lens[r], n = len[r];
    starts[r] = (int)min(row, (long long)INT32_MAX);
    if (n == REFUSED) {
      code = min(code, LOCRET_ERR_INVALID);
    } else if (x > 0) {
      if ((long long)n + x > room || row + x > a.n_tok) {
        len[r] = REFUSED;
        code = min(code, LOCRET_ERR_CAPACITY);
      } else {
        need += pages_of((long long)n + x) - pages_of(n);
      }
    }
    row += max(x, 0);
  }
  long long want = block_scan(need, warp_sums, &total_need);
  for (int r = r0; r < r1; r++) {
    const int x = a.new_lens[r], n = len[r];
    need0[r] = (int)min(want, (long long)top);
    if (n == REFUSED || x <= 0) continue;
    const int more = pages_of((long long)n + x) - pages_of(n);
    want += more;
    if (more > 0 && want > top) {   // (and so is every later request that needs a page)
      len[r] = REFUSED;
      need0[r] = top;
      code = min(code, LOCRET_ERR_CAPACITY);
    }
  }
  if (tid == 0) {
    starts[a.n_req] = (int)min(total_rows, (long long)INT32_MAX);
    if (bad_list || too_many) code = min(code, LOCRET_ERR_INVALID);
  }
  if (code && rank == 0) report(a.status, code);

  // ended requests: their pages onto the list, one warp for each request, over all blocks
  for (int r = r0; __any_sync(0xffffffffu, r < r1); r++) {
    int count = 0, at = 0;
    if (r < r1 && a.new_lens[r] < 0 && len[r] != REFUSED) {
      count = pages_of(len[r]);
      at = (int)min(push, (long long)INT32_MAX);
      push += count;
    }
    for (unsigned todo = __ballot_sync(0xffffffffu, count > 0); todo; todo &= todo - 1) {
      const int src = __ffs(todo) - 1;
      const int c = __shfl_sync(0xffffffffu, count, src), first = __shfl_sync(0xffffffffu, at, src),
                rr = __shfl_sync(0xffffffffu, r, src);
      for (int j = rank * 32 + (tid & 31); j < c; j += n_blocks * 32) {
        const long long to = (long long)n_free + first + j;
        if (to < a.capacity) a.free_pages[to] = a.table[rr * a.table_stride + j];
      }
    }
  }
  // Number of pages taken: the requests that get theirs come before the first that does not.
  __shared__ int taken;
  if (tid == 0) taken = 0;
  __syncthreads();
  {
    int last = 0;
    for (int r = r0; r < r1; r++)
      if (len[r] != REFUSED && a.new_lens[r] > 0) {
        const int more = pages_of((long long)len[r] + a.new_lens[r]) - pages_of(len[r]);
        if (more > 0) last = max(last, need0[r] + more);
      }
    last = __reduce_max_sync(0xffffffffu, last);
    if ((tid & 31) == 0) atomicMax(&taken, last);
  }
  __syncthreads();
  const int n_taken = taken;
  if (tid == 0) need0[a.n_req] = n_taken;
  // a request behind the last one that takes pages begins where the list's part ends
  for (int r = r0; r < r1; r++) need0[r] = min(need0[r], n_taken);

  // everything that is read has been read, and what was pushed can be seen
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");

  for (int r = rank * PS_THREADS + tid; r < a.n_req; r += n_blocks * PS_THREADS) {
    const int x = a.new_lens[r];
    a.starts[r] = starts[r];
    if (len[r] == REFUSED) {
      if (a.lens_out != a.lens_in) a.lens_out[r] = a.lens_in[r];
    } else {
      a.lens_out[r] = x < 0 ? 0 : len[r] + x;
    }
  }
  if (rank == 0 && tid == 0) {
    a.starts[a.n_req] = starts[a.n_req];
    *a.n_free_out = top - n_taken;
  }
  // the table's new entries
  for (int k = rank * PS_THREADS + tid; k < n_taken; k += n_blocks * PS_THREADS) {
    const int r = owner(need0, a.n_req, k);
    a.table[r * a.table_stride + pages_of(len[r]) + k - need0[r]] = a.free_pages[top - 1 - k];
  }
  // the rows
  const int n_rows = starts[a.n_req];
  for (int t = rank * PS_THREADS + tid; t < a.n_tok; t += n_blocks * PS_THREADS) {
    int64_t slot = -1;
    int pos = 0;
    if (t < n_rows) {
      const int r = owner(starts, a.n_req, t), n = len[r];
      if (n != REFUSED) {
        pos = n + (t - starts[r]);
        const int j = pos / page, old = pages_of(n);
        const int p = j < old ? a.table[r * a.table_stride + j] : a.free_pages[top - 1 - (need0[r] + j - old)];
        if (p >= 0 && p < a.capacity) slot = (int64_t)p * page + (pos - j * page);
        else report(a.status, LOCRET_ERR_INVALID);
      } else {
        pos = (int)max(0LL, min((long long)a.lens_in[r] + (t - starts[r]), (long long)INT32_MAX));
      }
    }
    a.slots[t] = slot;
    a.positions[t] = pos;
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
  const int p = pos >= 0 && pos < len ? table[pos / pg.page_size] : -1;
  if (p < 0 || p >= pg.n_pages) { report(status, LOCRET_ERR_INVALID); return; }
  const size_t src = ((size_t)m * cap + i) * d + c;
  const long long dst = p * pg.page_stride + m * pg.head_stride + (pos % pg.page_size) * pg.token_stride + c;
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

extern "C" int locret_pages_step(int32_t *table, int64_t table_stride, int32_t width, const int32_t *lens_in, int32_t *lens_out,
                                 const int32_t *new_lens, int32_t n_req, int32_t page_size, int32_t *free_pages,
                                 int32_t capacity, const int32_t *n_free_in, int32_t *n_free_out, int32_t n_tok, int64_t *slots,
                                 int32_t *positions, int32_t *starts, int32_t *status, void *stream) {
  if (n_req < 0 || n_req > LOCRET_MAX_REQUESTS || n_tok < 0 || page_size < 1 || width < 1 || capacity < 1 || table_stride < 0)
    return LOCRET_ERR_INVALID;
  if (!free_pages || !n_free_in || !n_free_out || !starts || (n_tok && (!slots || !positions))) return LOCRET_ERR_INVALID;
  if (n_req && (!table || !lens_in || !lens_out || !new_lens || (n_req > 1 && table_stride < width))) return LOCRET_ERR_INVALID;
  const PagesStepArgs a = {table, table_stride, lens_in, new_lens, n_free_in, lens_out, free_pages, n_free_out, positions,
                           starts, status, slots, width, n_req, page_size, capacity, n_tok};
  cudaLaunchConfig_t cfg = {};
  const int work = n_tok > n_req ? n_tok : n_req;
  int blocks = 1;   // (a power of two, so that clusters of it exist)
  while (blocks < PS_MAX_BLOCKS && blocks * PS_THREADS < work) blocks *= 2;
  const size_t smem = sizeof(int) * (3 * (size_t)n_req + 2);
  static PerDeviceFlag flag;
  if (allow_dynamic_smem(pages_step_kernel, (int)sizeof(int) * (3 * LOCRET_MAX_REQUESTS + 2), flag) != cudaSuccess) {
    cudaGetLastError();
    return LOCRET_ERR_CUDA;
  }
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(PS_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = (cudaStream_t)stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = blocks;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, pages_step_kernel, a) != cudaSuccess) { cudaGetLastError(); return LOCRET_ERR_CUDA; }
  return LOCRET_OK;
}
