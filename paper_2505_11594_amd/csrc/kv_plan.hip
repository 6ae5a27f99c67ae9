// Page tables and slots of a batch of requests, from their lengths: pages of requests that
// have ended go back on the stack of free pages, requests that bring tokens take theirs from
// it, and every new token gets its position and its slot in the cache.  Whole numbers
// only; what it takes is the way through memory and the launches: 7 us for the next step of 256
// requests of up to 8000 cached tokens, a tenth of them ended; 6 + 4 us for 64 prompts of up to 2000 tokens.
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

// Sums that stop at 2^32 - 1: what is larger is compared with counts below 2^31 only.
struct Pair {
  uint32_t x, y;
};
__device__ __forceinline__ Pair add(Pair a, Pair b) {
  return Pair{__builtin_elementwise_add_sat(a.x, b.x), __builtin_elementwise_add_sat(a.y, b.y)};
}
template <int CTRL, int ROWS>
__device__ __forceinline__ Pair add_dpp(Pair a) {        // lanes that the control does not reach add 0
  return add(a, Pair{(uint32_t)__builtin_amdgcn_update_dpp(0, (int)a.x, CTRL, ROWS, 0xF, false),
                     (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a.y, CTRL, ROWS, 0xF, false)});
}
__device__ __forceinline__ Pair row_scan(Pair a) {       // over the lanes of a row of 16 up to this one
  a = add_dpp<0x111, 0xF>(a);
  a = add_dpp<0x112, 0xF>(a);
  a = add_dpp<0x114, 0xF>(a);
  return add_dpp<0x118, 0xF>(a);
}
// Sums over the threads up to this one, and over all; the next call takes the other `red`
// (of PT / 64 entries each), so that one barrier does.
__device__ __forceinline__ Pair scan(Pair v, Pair* red, Pair* all) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  v = row_scan(v);
  v = add_dpp<0x142, 0xA>(v);                            // lane 15 of a row to the next, lane 31 to the upper half
  v = add_dpp<0x143, 0xC>(v);
  if (lane == 63) red[wave] = v;
  __syncthreads();
  const Pair w = row_scan(red[lane & 15]);
  *all = Pair{(uint32_t)__builtin_amdgcn_readlane((int)w.x, 15), (uint32_t)__builtin_amdgcn_readlane((int)w.y, 15)};
  if (wave == 0) return v;
  return add(v, Pair{(uint32_t)__builtin_amdgcn_readlane((int)w.x, wave - 1), (uint32_t)__builtin_amdgcn_readlane((int)w.y, wave - 1)});
}
static_assert(PT == 1024, "a row of lanes holds the waves' sums");

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
//
// What it takes is latency: loads that wait for one another, barriers.  So a thread loads its
// request once for both passes (where one thread has one), and the page that its next token may
// go to before it is known whether it does; and where no request brings more than DIRECT pages or
// tokens -- every batch that generates -- it writes them itself, without the search.  (256 requests:
// 27 us with 64-bit scans through shuffles, every request loaded twice, and searches.)
constexpr int DIRECT = 2;
template <bool INLINE>
__global__ __launch_bounds__(PT) void plan_kernel(const Plan a) {
  __shared__ Pair red[2][PT / 64];
  __shared__ int seq[PT], len[PT], tok0[PT], page0[PT];
  __shared__ uint32_t first[PT];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int capacity = a.max_pages * a.page_size;
  const uint32_t most = (uint32_t)a.free_capacity;
  uint32_t avail = (uint32_t)imax(0, imin(*a.n_free, a.free_capacity));
  int count = 0, had = 0, held = 0, last = -1;           // of this thread's request; last: the page of token `had`, if held
  auto fetch = [&](int s) {
    count = s < a.S ? a.counts[s] : 0;
    had = s < a.S ? cached_len(a.lens[s], capacity) : 0;
    held = cdiv(had, a.page_size);
    last = -1;
    if (INLINE && s < a.S && had / a.page_size < held) last = a.table[(size_t)s * a.max_pages + had / a.page_size];
  };

  // pages of requests that have ended
  for (int s0 = 0; s0 < a.S; s0 += PT) {
    const int s = s0 + tid;
    fetch(s);
    const bool ended = count < 0;
    Pair all;
    const Pair at = scan(Pair{ended, ended ? (uint32_t)held : 0u}, red[0], &all);
    if (all.x == 0) {
      __syncthreads();                                   // (red is written again)
      continue;
    }
    if (ended) {
      seq[at.x - 1] = s;
      len[at.x - 1] = held;
      first[at.x - 1] = add(Pair{avail, 0}, Pair{at.y, 0}).x - (uint32_t)held;
    }
    __syncthreads();
    for (int r = wave; r < (int)all.x; r += PT / 64) {   // a wave to a request
      int32_t* const row = a.table + (size_t)seq[r] * a.max_pages;
      const int n = len[r];
      const uint32_t to = first[r];
      for (int j0 = 0; j0 < a.max_pages; j0 += 512) {
        int page[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) page[u] = row[imin(j0 + 64 * u + lane, a.max_pages - 1)];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int j = j0 + 64 * u + lane;
          if (j < a.max_pages) row[j] = -1;
          if (j < n && to < most && (uint32_t)j < most - to) a.free_pages[to + j] = page[u];
        }
      }
    }
    avail = min(add(Pair{avail, 0}, Pair{all.y, 0}).x, most);
    __syncthreads();
  }

  // requests that bring tokens
  Pair asked{0, 0};
  uint32_t taken = 0, total = 0;
  for (int s0 = 0; s0 < a.S; s0 += PT) {
    const int s = s0 + tid;
    if (a.S > PT) fetch(s);
    if (count < 0) had = held = 0;
    const bool able = count > 0 && count <= capacity - had;
    const int need = able ? cdiv(had + count, a.page_size) - held : 0;
    Pair all;
    const Pair upto = add(asked, scan(Pair{(uint32_t)need, able ? (uint32_t)count : 0u}, red[0], &all));
    asked = add(asked, all);
    const bool ok = able && (need == 0 || upto.x <= avail) && upto.y <= (uint32_t)a.max_tokens;
    const int granted = ok ? count : 0, pages = ok ? need : 0;
    Pair sum;
    const Pair got = scan(Pair{(uint32_t)pages, (uint32_t)granted}, red[1], &sum);
    const uint32_t t0 = total + got.y - (uint32_t)granted, top = avail - 1 - (upto.x - (uint32_t)need);   // its first page's place
    if (s < a.S) {
      a.granted[s] = granted;
      a.starts[s] = (int)t0;
      a.lens[s] = had + granted;
    }
    if (__syncthreads_or(pages > DIRECT || granted > DIRECT)) {
      seq[tid] = s;
      len[tid] = had;
      first[tid] = top;
      page0[tid] = (int)(got.x - (uint32_t)pages);
      tok0[tid] = (int)(got.y - (uint32_t)granted);
      __syncthreads();
      for (int i = tid; i < (int)sum.x; i += PT) {       // new pages, each found by its place in the scan
        const int r = last_at_most(page0, PT, i), j = i - page0[r];
        a.table[(size_t)seq[r] * a.max_pages + cdiv(len[r], a.page_size) + j] = a.free_pages[first[r] - (uint32_t)j];
      }
      if constexpr (INLINE) {
        for (int i = tid; i < (int)sum.y; i += PT) {
          const int r = last_at_most(tok0, PT, i), p = len[r] + i - tok0[r], j = p / a.page_size - cdiv(len[r], a.page_size);
          const int page = j >= 0 ? a.free_pages[first[r] - (uint32_t)j] : a.table[(size_t)seq[r] * a.max_pages + p / a.page_size];
          store_token(a, (long long)total + i, p, page);
        }
      }
    } else {
      int page[DIRECT];
#pragma unroll
      for (int j = 0; j < DIRECT; ++j)
        if (j < pages) {
          page[j] = a.free_pages[top - (uint32_t)j];
          a.table[(size_t)s * a.max_pages + held + j] = page[j];
        }
      if constexpr (INLINE) {
#pragma unroll
        for (int i = 0; i < DIRECT; ++i)
          if (i < granted) {
            const int j = (had + i) / a.page_size - held;
            store_token(a, (long long)t0 + i, had + i, j < 0 ? last : page[j > 0 ? 1 : 0]);
          }
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
    for (long long i = (long long)total + tid; i < a.max_tokens; i += PT) {
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
