// Page tables and slots of a batch of requests, from their lengths: pages of requests that
// have ended go back on the stack of free pages, requests that bring tokens take theirs from
// it, and every new token gets its position and its slot in the cache.  Whole numbers
// only; what it takes is the way through memory and the launches.
//
// Requests are granted in their order: with A and C the sums of the pages and tokens asked
// for up to a request, its own among them (by requests that cannot fit their row of the table:
// none), it is granted iff (it needs no page or A <= free pages) and C <= max_tokens.  Sums of
// what was asked, not of what was granted: so a scan gives all answers at once, the granted
// ones that need pages are the first ones, and their pages lie behind one another on the stack.
#include "lm_args.h"
#include "window.h"

namespace sage {

constexpr int PT = 1024;                                 // threads of the one workgroup that scans

struct Scan {
  long long x, y;
};
// Sums over the threads before this one; `all` of every thread.  red: 2 * PT / 64 entries.
__device__ __forceinline__ Scan scan_before(long long x, long long y, Scan* red, Scan* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Scan s{x, y};
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long px = __shfl_up(s.x, o, 64), py = __shfl_up(s.y, o, 64);
    if (lane >= o) { s.x += px; s.y += py; }
  }
  __syncthreads();                                       // (red may still be read from the last call)
  if (lane == 63) red[wave] = s;
  __syncthreads();
  Scan before{0, 0};
  *all = Scan{0, 0};
#pragma unroll
  for (int w = 0; w < PT / 64; ++w) {
    const Scan r = red[w];
    if (w < wave) { before.x += r.x; before.y += r.y; }
    all->x += r.x;
    all->y += r.y;
  }
  return Scan{before.x + s.x - x, before.y + s.y - y};
}

// The last of n ascending entries that is at most x (the first one is).
__device__ __forceinline__ int last_at_most(const int* at, int n, int x) {
  int lo = 0;
  while (n > 1) {
    const int half = n / 2;
    if (at[lo + half] <= x) { lo += half; n -= half; }
    else n = half;
  }
  return lo;
}

__device__ __forceinline__ void store_token(const Plan& a, long long i, int at, int page) {
  a.pos[i] = at;
  a.slots[i] = (long long)page * a.page_size + at % a.page_size;
}

// INLINE: the new tokens' places too, by the same workgroup.
template <bool INLINE>
__global__ __launch_bounds__(PT) void plan_kernel(const Plan a) {
  __shared__ Scan red[PT / 64];
  __shared__ int seq[PT], len[PT], tok0[PT], page0[PT];
  __shared__ long long first[PT];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int capacity = a.max_pages * a.page_size;
  long long avail = imax(0, imin(*a.n_free, a.free_capacity));

  // pages of requests that have ended
  for (int s0 = 0; s0 < a.S; s0 += PT) {
    const int s = s0 + tid;
    const bool ended = s < a.S && a.counts[s] < 0;
    const int held = ended ? cdiv(cached_len(a.lens[s], capacity), a.page_size) : 0;
    Scan all;
    const Scan at = scan_before(ended, held, red, &all);
    if (ended) {
      seq[at.x] = s;
      len[at.x] = held;
      first[at.x] = avail + at.y;
    }
    __syncthreads();
    for (int r = wave; r < (int)all.x; r += PT / 64) {   // a wave to a request
      int32_t* const row = a.table + (size_t)seq[r] * a.max_pages;
      for (int j0 = 0; j0 < a.max_pages; j0 += 256) {
        int page[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) page[u] = row[imin(j0 + 64 * u + lane, a.max_pages - 1)];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int j = j0 + 64 * u + lane;
          if (j >= a.max_pages) continue;
          row[j] = -1;
          if (j < len[r] && first[r] + j < a.free_capacity) a.free_pages[first[r] + j] = page[u];
        }
      }
    }
    avail = avail + all.y < a.free_capacity ? avail + all.y : a.free_capacity;
    __syncthreads();
  }

  // requests that bring tokens
  long long asked_pages = 0, asked_tokens = 0, taken = 0, total = 0;
  for (int s0 = 0; s0 < a.S; s0 += PT) {
    const int s = s0 + tid;
    const int count = s < a.S ? a.counts[s] : 0;
    const int had = s < a.S && count >= 0 ? cached_len(a.lens[s], capacity) : 0;
    const bool able = count > 0 && count <= capacity - had;
    const int held = cdiv(had, a.page_size), need = able ? cdiv(had + count, a.page_size) - held : 0;
    Scan all;
    const Scan asked = scan_before(need, able ? count : 0, red, &all);
    const long long before = asked_pages + asked.x;
    const bool ok = able && (need == 0 || before + need <= avail) && asked_tokens + asked.y + count <= a.max_tokens;
    asked_pages += all.x;
    asked_tokens += all.y;
    const int granted = ok ? count : 0;
    Scan sum;
    const Scan at = scan_before(ok ? need : 0, granted, red, &sum);
    if (s < a.S) {
      a.granted[s] = granted;
      a.starts[s] = (int)(total + at.y);
      a.lens[s] = had + granted;
    }
    seq[tid] = s;
    len[tid] = had;
    first[tid] = before;
    page0[tid] = (int)at.x;
    tok0[tid] = (int)at.y;
    __syncthreads();
    for (int i = tid; i < (int)sum.x; i += PT) {         // new pages, each found by its place in the scan
      const int r = last_at_most(page0, PT, i), j = i - page0[r];
      a.table[(size_t)seq[r] * a.max_pages + cdiv(len[r], a.page_size) + j] = a.free_pages[avail - 1 - (first[r] + j)];
    }
    if constexpr (INLINE) {
      for (int i = tid; i < (int)sum.y; i += PT) {
        const int r = last_at_most(tok0, PT, i), p = len[r] + i - tok0[r], j = p / a.page_size - cdiv(len[r], a.page_size);
        const int page = j >= 0 ? a.free_pages[avail - 1 - (first[r] + j)] : a.table[(size_t)seq[r] * a.max_pages + p / a.page_size];
        store_token(a, total + i, p, page);
      }
    }
    taken += sum.x;
    total += sum.y;
    __syncthreads();
  }
  if (tid == 0) {
    a.starts[a.S] = (int)total;
    *a.n_free = (int)(avail - taken);
  }
  if constexpr (INLINE) {
    for (long long i = total + tid; i < a.max_tokens; i += PT) {
      a.pos[i] = 0;
      a.slots[i] = -1;
    }
  }
}

// The new tokens' places, from the tables and lengths that plan_kernel left.
__global__ __launch_bounds__(256) void plan_tokens_kernel(const Plan a) {
  const int total = a.starts[a.S];
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < a.max_tokens; i += (long long)gridDim.x * 256) {
    if (i >= total) {
      a.pos[i] = 0;
      a.slots[i] = -1;
      continue;
    }
    const int s = last_at_most(a.starts, a.S, (int)i);
    const int p = a.lens[s] - a.granted[s] + (int)i - a.starts[s];
    store_token(a, i, p, a.table[(size_t)s * a.max_pages + p / a.page_size]);
  }
}

hipError_t launch_kv_plan(const Plan& a, hipStream_t st) {
  if (a.max_tokens <= 4 * PT) {
    hipLaunchKernelGGL(plan_kernel<true>, dim3(1), dim3(PT), 0, st, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(plan_kernel<false>, dim3(1), dim3(PT), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int blocks = cdiv(a.max_tokens, 256);
  hipLaunchKernelGGL(plan_tokens_kernel, dim3((unsigned)imin(blocks, 4096)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace sage
