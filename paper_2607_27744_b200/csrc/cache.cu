// Paged cache of request histories: handle, bookkeeping of pages (extend, fork, truncate, compact) and the writing of
// new rows.
//
// Books are kept by one CTA: which pages are free, whose turn each is and whether the call can be carried out at all is a
// chain of prefix sums over the slots of the call and the holders of all pages, a few thousand integers from L2.  It
// leaves what is to be moved as a list in the workspace; a second kernel, launched behind it as a programmatic dependent,
// moves the bytes on the whole chip.  Nothing depends on the order of atomics: they count holders and keep the largest
// status; pages are dealt out by prefix sums, and the order of the list of copies does not matter.
#include <algorithm>
#include <new>

#include "cache.h"
#include "sm100_ptx.cuh"

namespace rocs {
namespace {

constexpr int kBookThreads = 1024;
constexpr int32_t kOk = 0, kFewPages = 1, kBadSlot = 2, kTooLong = 3, kNotEmpty = 4, kBadPage = 5;
// Entries (slots x width) up to which the CTA that checks a fork or truncate also carries it out: a second launch is about
// 2 us, one CTA takes about 1 us per 2048 entries.
constexpr int64_t kOneCtaEntries = 8192;

// Workspace in int32 words: head, then arrays of n_slots, n + 1, n + 1, n_pages, n_pages, n_pages words.
struct Books {
  int32_t* head;    // [0] status, [1] entries of the call, [2] pairs to copy
  int32_t* owner;   // [n_slots] the call's index that names a slot
  int32_t* before;  // [n + 1] entries in front of an index
  int32_t* start;   // [n] first column of an index's entries (truncate, extend) or length (fork)
  int32_t* src;     // [n_pages] pages to copy from (extend: behind the free list)
  int32_t* dst;     // [n_pages] pages to copy to
  int32_t* map;     // [n_pages] free list (extend), new place of a page (compact)
};
__host__ __device__ inline size_t books_words(int32_t n_slots, int32_t n, int32_t n_pages) {
  return 16 + (size_t)n_slots + 2 * ((size_t)n + 1) + 3 * (size_t)n_pages;
}
Books books_in(void* workspace, const rocs_cache* c, int32_t n) {
  Books b;
  b.head = static_cast<int32_t*>(workspace);
  b.owner = b.head + 16;
  b.before = b.owner + c->n_slots;
  b.start = b.before + n + 1;
  b.src = b.start + n + 1;
  b.dst = b.src + c->n_pages;
  b.map = b.dst + c->n_pages;
  return b;
}

struct CacheBooks {
  int32_t n_pages, page, n_slots, width;
  int32_t *table, *lens, *refs;
};
CacheBooks books_of(const rocs_cache* c) {
  return CacheBooks{c->n_pages, c->page, c->n_slots, c->width, c->table, c->lens, c->refs};
}

// Exclusive prefix sum of one value per thread over the CTA, and the total; all threads call it.
__device__ __forceinline__ int32_t block_prefix(int32_t v, int32_t& total) {
  __shared__ int32_t sums[kBookThreads / 32];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  int32_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int32_t up = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += up;
  }
  __syncthreads();  // the sums of the call in front have been read
  if (lane == 31) sums[warp] = incl;
  __syncthreads();
  int32_t s = sums[lane];  // 32 warps
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int32_t up = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += up;
  }
  total = __shfl_sync(0xffffffffu, s, 31);
  const int32_t base = __shfl_sync(0xffffffffu, s, (warp + 31) % 32);
  return incl - v + (warp > 0 ? base : 0);
}

// A bit per slot in shared memory for as many slots as fit, otherwise a word per slot in the workspace.
constexpr int32_t kBitSlots = 32 * 8192;
struct Claims {
  uint32_t* bits;  // null: by `owner`
  int32_t* owner;
};
// Clears what claim() uses; a barrier follows.
__device__ __forceinline__ void clear_claims(const CacheBooks& c, const Claims& k, const int32_t* slots, int32_t n) {
  if (k.bits) {
    for (int32_t x = threadIdx.x; x < (c.n_slots + 31) / 32; x += kBookThreads) k.bits[x] = 0;
  } else {
    for (int32_t i = threadIdx.x; i < n; i += kBookThreads) {
      const int32_t s = slots ? slots[i] : i;
      if (s >= 0 && s < c.n_slots) k.owner[s] = 0;
    }
  }
  __syncthreads();
}
// false: the slot is none, or has been named by the call already.
__device__ __forceinline__ bool claim(const CacheBooks& c, const Claims& k, int32_t s) {
  if (s < 0 || s >= c.n_slots) return false;
  if (k.bits) return (atomicOr(k.bits + s / 32, 1u << (s % 32)) >> (s % 32) & 1u) == 0;
  return atomicExch(k.owner + s, 1) == 0;
}

// The index whose entries entry f is among: largest i with before[i] <= f.
__device__ __forceinline__ int32_t index_of(const int32_t* before, int32_t n, int32_t f) {
  int32_t lo = 0, hi = n;
  while (hi - lo > 1) {
    const int32_t mid = lo + (hi - lo) / 2;
    if (before[mid] <= f) lo = mid; else hi = mid;
  }
  return lo;
}

__device__ __forceinline__ int32_t load_flags(const int32_t* refs, int32_t n_pages, int32_t first, int32_t (&v)[4]) {
  if (first + 4 <= n_pages) {  // refs is 16-byte aligned and first a multiple of 4
    const int4 x = *reinterpret_cast<const int4*>(refs + first);
    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
    return 4;
  }
  const int32_t m = max(n_pages - first, 0);
  for (int k = 0; k < 4; ++k) v[k] = k < m ? refs[first + k] : 0;
  return m;
}

constexpr int32_t kNearPages = 4 * kBookThreads;  // free pages that are kept in shared memory

__global__ void __launch_bounds__(kBookThreads, 1)
extend_kernel(CacheBooks c, const int32_t* slots, const int32_t* off, int32_t R, Books b, int32_t* first, int32_t* report) {
  extern __shared__ uint32_t bits[];
  __shared__ int32_t status, copies, near_before[kBookThreads + 1], near_place[kBookThreads], near_free[kNearPages];
  const Claims claims{c.n_slots <= kBitSlots ? bits : nullptr, b.owner};
  const bool near = R <= kBookThreads;  // the requests' places are kept in shared memory
  if (threadIdx.x == 0) { status = kOk; copies = 0; }
  ptx::griddep_wait_for(slots, off);
  ptx::griddep_launch_dependents();
  // the first pages' holders, long before they are asked for
  int32_t v[4], m = load_flags(c.refs, c.n_pages, 4 * (int32_t)threadIdx.x, v);
  clear_claims(c, claims, slots, R);
  // pages that each request needs
  int64_t total64 = 0;
  int32_t my_slot = 0, my_n = 0, my_L = 0, my_start = 0;  // of the last request that this thread looked at
  for (int32_t r0 = 0; r0 < R; r0 += kBookThreads) {
    const int32_t r = r0 + (int32_t)threadIdx.x;
    int32_t need = 0;
    if (r < R) {
      const int32_t s = slots ? slots[r] : r, n = off[r + 1] - off[r];
      my_slot = s;
      my_n = n;
      if (!claim(c, claims, s)) {
        atomicMax(&status, kBadSlot);
      }
      if (s >= 0 && s < c.n_slots) {
        const int32_t L = c.lens[s];
        my_L = L;
        if (L < 0 || (int64_t)L + n > (int64_t)c.width * c.page) {
          atomicMax(&status, kTooLong);
        } else if (n > 0) {
          bool copy = false;
          if (L % c.page != 0) {
            const int32_t id = c.table[(int64_t)s * c.width + L / c.page];
            if (id < 0 || id >= c.n_pages) atomicMax(&status, kBadPage);
            else copy = c.refs[id] > 1;
          }
          my_start = pages_for(L, c.page) - (copy ? 1 : 0);
          need = pages_for(L + n, c.page) - my_start;
        } else {
          my_start = pages_for(L, c.page);
        }
      }
    }
    int32_t sum;
    const int32_t at = block_prefix(need, sum);
    if (r < R) {
      if (near) {
        near_before[r] = (int32_t)(total64 + at);
        near_place[r] = my_start;
      } else {
        b.before[r] = (int32_t)(total64 + at);
        b.start[r] = my_start;
      }
    }
    total64 += sum;
  }
  // That many free pages, lowest first.  (What the call needs may be beyond the pool and beyond 32 bits: then all free ones are
  // counted, and nothing is dealt out.)
  const int32_t total = (int32_t)min(total64, (int64_t)c.n_pages + 1);
  int32_t found = 0;
  for (int32_t p0 = 0; p0 < c.n_pages && found < total; p0 += 4 * kBookThreads) {
    const int32_t p = p0 + 4 * (int32_t)threadIdx.x;
    if (p0 > 0) m = load_flags(c.refs, c.n_pages, p, v);
    int32_t mine = 0, sum;
    for (int k = 0; k < 4; ++k) mine += k < m && v[k] == 0;
    int32_t at = found + block_prefix(mine, sum);
    for (int k = 0; k < 4; ++k)
      if (k < m && v[k] == 0) {
        if (at < kNearPages) near_free[at] = p + k;
        else if (at < total) b.map[at] = p + k;
        ++at;
      }
    found += sum;
  }
  __syncthreads();
  if (threadIdx.x == 0 && status == kOk && found < total) status = kFewPages;
  __syncthreads();
  const bool ok = status == kOk;
  if (threadIdx.x == 0) {
    b.head[0] = status;
    if (report) {
      report[0] = status;
      report[1] = ok ? total : status == kFewPages ? (int32_t)min(total64 - found, (int64_t)0x7fffffff) : 0;
    }
  }
  if (!ok) {
    for (int32_t r = threadIdx.x; r < R; r += kBookThreads) first[r] = -1;
    if (threadIdx.x == 0) b.head[2] = 0;
    return;
  }
  const int32_t* before = near ? near_before : b.before;
  const int32_t* place = near ? near_place : b.start;
  auto free_page = [&](int32_t f) { return f < kNearPages ? near_free[f] : b.map[f]; };
  // shared last pages: from there the row is a copy's; their entries are still the old ones
  for (int32_t r = threadIdx.x; r < R; r += kBookThreads) {
    if (!near) {
      my_slot = slots ? slots[r] : r;
      my_n = off[r + 1] - off[r];
      my_L = c.lens[my_slot];
      my_start = place[r];
    }
    first[r] = my_L;
    if (my_n > 0 && my_start < pages_for(my_L, c.page)) {
      const int32_t id = c.table[(int64_t)my_slot * c.width + my_start], at = atomicAdd(&copies, 1);
      b.src[at] = id;
      b.dst[at] = free_page(before[r]);
      atomicSub(c.refs + id, 1);
    }
    c.lens[my_slot] = my_L + my_n;
  }
  __syncthreads();
  if (threadIdx.x == 0) b.head[2] = copies;
  for (int32_t f = threadIdx.x; f < total; f += kBookThreads) {
    const int32_t r = index_of(before, R, f), s = slots ? slots[r] : r, id = free_page(f);
    c.table[(int64_t)s * c.width + place[r] + (f - before[r])] = id;
    c.refs[id] = 1;
  }
}

// A fork's or truncate's entries, carried out by `threads` threads of which this is number `thread`.
__device__ void apply_fork(const CacheBooks& c, const int32_t* parents, const int32_t* children, int32_t n, const Books& b,
                           int32_t total, int32_t thread, int32_t threads) {
  for (int32_t f = thread; f < total; f += threads) {
    const int32_t i = index_of(b.before, n, f), k = f - b.before[i];
    const int32_t id = c.table[(int64_t)parents[i] * c.width + k];
    c.table[(int64_t)children[i] * c.width + k] = id;
    if (id >= 0 && id < c.n_pages) atomicAdd(c.refs + id, 1);
  }
}
__device__ void apply_truncate(const CacheBooks& c, const int32_t* slots, int32_t n, const Books& b, int32_t total, int32_t thread,
                               int32_t threads) {
  for (int32_t f = thread; f < total; f += threads) {
    const int32_t i = index_of(b.before, n, f), k = b.start[i] + f - b.before[i];
    const int32_t id = c.table[(int64_t)slots[i] * c.width + k];
    if (id >= 0 && id < c.n_pages) atomicSub(c.refs + id, 1);
  }
}

// parents == NULL: truncate `slots` to `keep`; otherwise fork parents into `slots`.
__global__ void __launch_bounds__(kBookThreads, 1)
check_kernel(CacheBooks c, const int32_t* parents, const int32_t* slots, const int32_t* keep, int32_t n, Books b, int32_t* report,
             bool carry_out) {
  extern __shared__ uint32_t bits[];
  __shared__ int32_t status, near_before[kBookThreads + 1], near_place[kBookThreads];
  const Claims claims{c.n_slots <= kBitSlots ? bits : nullptr, b.owner};
  const bool near = carry_out && n <= kBookThreads;  // the slots' places are kept in shared memory
  if (near) {
    b.before = near_before;
    b.start = near_place;
  }
  if (threadIdx.x == 0) status = kOk;
  ptx::griddep_wait_for(parents, slots, keep);
  ptx::griddep_launch_dependents();
  clear_claims(c, claims, slots, n);
  int64_t total64 = 0;
  for (int32_t i0 = 0; i0 < n; i0 += kBookThreads) {
    const int32_t i = i0 + (int32_t)threadIdx.x;
    int32_t entries = 0;
    if (i < n) {
      const int32_t s = slots[i];
      if (!claim(c, claims, s)) atomicMax(&status, kBadSlot);
      if (s >= 0 && s < c.n_slots) {
        const int32_t L = c.lens[s];
        if (parents) {
          const int32_t q = parents[i];
          if (q < 0 || q >= c.n_slots || q == s) {
            atomicMax(&status, kBadSlot);
          } else {
            const int32_t Lq = c.lens[q];
            if (L != 0) atomicMax(&status, kNotEmpty);
            if (Lq < 0 || Lq > (int64_t)c.width * c.page) atomicMax(&status, kTooLong);
            else entries = pages_for(Lq, c.page);
            b.start[i] = Lq;
          }
        } else if (L < 0 || L > (int64_t)c.width * c.page) {
          atomicMax(&status, kTooLong);
        } else {
          const int32_t left = min(max(keep ? keep[i] : 0, 0), L);
          b.start[i] = pages_for(left, c.page);
          entries = pages_for(L, c.page) - b.start[i];
        }
      }
    }
    int32_t sum;
    const int32_t at = block_prefix(entries, sum);
    if (i < n) b.before[i] = (int32_t)(total64 + at);
    total64 += sum;
    if (total64 > 0x3fffffff) {
      atomicMax(&status, kTooLong);
      total64 = 0x3fffffff;
    }
  }
  __syncthreads();
  const bool ok = status == kOk;
  const int32_t total = ok ? (int32_t)total64 : 0;
  if (threadIdx.x == 0) {
    b.before[n] = total;
    b.head[0] = status;
    b.head[1] = total;
    if (report) {
      report[0] = status;
      report[1] = total;
    }
  }
  if (!ok) return;
  __syncthreads();
  for (int32_t i = threadIdx.x; i < n; i += kBookThreads) {
    if (parents) c.lens[slots[i]] = b.start[i];
    else c.lens[slots[i]] = min(max(keep ? keep[i] : 0, 0), c.lens[slots[i]]);
  }
  if (!carry_out) return;
  if (parents) apply_fork(c, parents, slots, n, b, total, threadIdx.x, kBookThreads);
  else apply_truncate(c, slots, n, b, total, threadIdx.x, kBookThreads);
}

__global__ void __launch_bounds__(256) apply_kernel(CacheBooks c, const int32_t* parents, const int32_t* slots, int32_t n, Books b) {
  ptx::griddep_wait_for(parents, slots);
  ptx::griddep_launch_dependents();
  const int32_t total = b.head[1], thread = blockIdx.x * 256 + threadIdx.x, threads = gridDim.x * 256;
  if (parents) apply_fork(c, parents, slots, n, b, total, thread, threads);
  else apply_truncate(c, slots, n, b, total, thread, threads);
}

// Which pages move where: the k-th page in use behind the line to the k-th free one in front of it.
__global__ void __launch_bounds__(kBookThreads, 1) compact_kernel(CacheBooks c, Books b, int32_t* refs_out, int32_t* report) {
  ptx::griddep_wait_for(refs_out, report);
  ptx::griddep_launch_dependents();
  int32_t mine = 0, line;
  for (int32_t p0 = 0; p0 < c.n_pages; p0 += 4 * kBookThreads) {
    int32_t v[4];
    const int32_t m = load_flags(c.refs, c.n_pages, p0 + 4 * (int32_t)threadIdx.x, v);
    for (int k = 0; k < 4; ++k) mine += k < m && v[k] > 0;
  }
  block_prefix(mine, line);
  int32_t n_src = 0, n_dst = 0;
  for (int32_t p0 = 0; p0 < c.n_pages; p0 += 4 * kBookThreads) {
    int32_t v[4];
    const int32_t p = p0 + 4 * (int32_t)threadIdx.x, m = load_flags(c.refs, c.n_pages, p, v);
    int32_t s = 0, d = 0, sum_s, sum_d;
    for (int k = 0; k < 4; ++k) {
      s += k < m && v[k] > 0 && p + k >= line;
      d += k < m && v[k] <= 0 && p + k < line;
    }
    int32_t at_s = n_src + block_prefix(s, sum_s), at_d = n_dst + block_prefix(d, sum_d);
    for (int k = 0; k < 4 && k < m; ++k) {
      if (v[k] > 0 && p + k >= line) b.src[at_s++] = p + k;
      if (v[k] <= 0 && p + k < line) b.dst[at_d++] = p + k;
      if (p + k >= line) b.map[p + k] = p + k;
      if (refs_out != c.refs) refs_out[p + k] = v[k];
    }
    n_src += sum_s;
    n_dst += sum_d;
  }
  __syncthreads();
  for (int32_t i = threadIdx.x; i < n_src; i += kBookThreads) {  // n_src == n_dst
    const int32_t from = b.src[i], to = b.dst[i];
    b.map[from] = to;
    refs_out[to] = c.refs[from];
  }
  __syncthreads();
  for (int32_t i = threadIdx.x; i < n_src; i += kBookThreads) refs_out[b.src[i]] = 0;
  if (threadIdx.x == 0) {
    b.head[0] = kOk;
    b.head[1] = line;
    b.head[2] = n_src;
    if (report) {
      report[0] = kOk;
      report[1] = line;
    }
  }
}

// A page's bytes: `outer` x `inner` runs of `vecs` 16-byte vectors (dimensions that follow one another without a gap are
// one run), at the same places in K and in V.
struct PageShape {
  uint8_t *K, *V;
  int64_t layer_bytes, page_bytes, outer_bytes, inner_bytes;
  int32_t layers, outer, inner, vecs;
};

// Copies the listed pages, all layers, K and V, and (compact) rewrites the table.  Each CTA takes pieces of kChunk vectors;
// a thread has kBatch of them in flight, which is what keeps the memory busy: the loads are independent and long.
constexpr int kCopyThreads = 256, kBatch = 8, kChunk = kCopyThreads * kBatch;
__global__ void __launch_bounds__(kCopyThreads) copy_pages_kernel(PageShape g, CacheBooks c, Books b, int32_t* table_out) {
  ptx::griddep_wait_for(table_out);
  ptx::griddep_launch_dependents();
  if (b.head[0] != kOk) return;
  const int32_t pairs = b.head[2];
  const int32_t page_vecs = g.outer * g.inner * g.vecs, chunks = (page_vecs + kChunk - 1) / kChunk;
  const int64_t pieces = (int64_t)pairs * g.layers * 2 * chunks;
  for (int64_t x = blockIdx.x; x < pieces; x += gridDim.x) {
    const int32_t chunk = (int32_t)(x % chunks);
    int64_t y = x / chunks;
    uint8_t* base = (y % 2 ? g.V : g.K);
    y /= 2;
    base += (y % g.layers) * g.layer_bytes;
    const int32_t pair = (int32_t)(y / g.layers);
    const uint8_t* from = base + b.src[pair] * g.page_bytes;
    uint8_t* to = base + b.dst[pair] * g.page_bytes;
    uint4 v[kBatch];
    int64_t at[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int32_t e = chunk * kChunk + k * kCopyThreads + (int32_t)threadIdx.x;
      at[k] = -1;
      if (e < page_vecs) {
        const int32_t run = e / g.vecs;
        at[k] = (run / g.inner) * g.outer_bytes + (run % g.inner) * g.inner_bytes + (int64_t)(e % g.vecs) * 16;
        v[k] = *reinterpret_cast<const uint4*>(from + at[k]);
      }
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      if (at[k] >= 0) *reinterpret_cast<uint4*>(to + at[k]) = v[k];
  }
  if (table_out == nullptr) return;
  const int32_t line = b.head[1];
  const int64_t entries = (int64_t)c.n_slots * c.width;
  for (int64_t e = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; e < entries; e += (int64_t)gridDim.x * kCopyThreads) {
    const int32_t s = (int32_t)(e / c.width), k = (int32_t)(e % c.width), id = c.table[e];
    const int32_t held = min(max(c.lens[s], 0), c.width * c.page);
    const bool moved = k < pages_for(held, c.page) && id >= line && id < c.n_pages;
    if (moved) table_out[e] = b.map[id];
    else if (table_out != c.table) table_out[e] = id;
  }
}

// A warp per new row.
constexpr int kAhead = 4;  // 16-byte vectors of K and of V per lane
struct AppendArgs {
  CacheBooks c;
  const int32_t *slots, *off, *first;
  int32_t R;
  int64_t N;
  int32_t H_kv, vecs;  // 16-byte vectors of a head
  uint8_t *K, *V;      // of the layer
  int64_t page_bytes, token_bytes, head_bytes;
  const uint8_t *K_new, *V_new;
  int64_t new_token_bytes, new_head_bytes;
};
// The request that row i of the batch is of, found by a warp: 32 offsets at a time.
__device__ __forceinline__ int32_t request_of(const int32_t* off, int32_t R, int64_t i, int lane) {
  int32_t lo = 0, n = R;  // requests lo .. lo + n - 1 may have the row
  while (n > 1) {
    const int32_t step = (n + 31) / 32, at = lo + lane * step;
    const uint32_t begun = __ballot_sync(0xffffffffu, lane * step < n && off[at] <= i);  // (the first has)
    const int32_t last = 31 - __clz((int)begun);
    n = min(step, n - last * step);
    lo += last * step;
  }
  return lo;
}

__global__ void __launch_bounds__(256) append_kernel(AppendArgs a) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int lane = threadIdx.x % 32;
  const int32_t total = a.H_kv * a.vecs;
  for (int64_t i = (int64_t)blockIdx.x * 8 + threadIdx.x / 32; i < a.N; i += (int64_t)gridDim.x * 8) {
    // the row's values are on their way while its place is looked up
    const int64_t from = i * a.new_token_bytes;
    uint4 k[kAhead], v[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const int32_t e = lane + 32 * x, h = e / a.vecs, at = (e - h * a.vecs) * 16;
      if (e < total) {
        k[x] = *reinterpret_cast<const uint4*>(a.K_new + from + h * a.new_head_bytes + at);
        v[x] = *reinterpret_cast<const uint4*>(a.V_new + from + h * a.new_head_bytes + at);
      }
    }
    const int32_t r = request_of(a.off, a.R, i, lane);
    const int32_t s = a.slots ? a.slots[r] : r, first = a.first[r];
    if (s < 0 || s >= a.c.n_slots || first < 0) continue;
    const int64_t pos = (int64_t)first + (i - a.off[r]);
    if (pos >= (int64_t)a.c.width * a.c.page) continue;
    const int32_t id = a.c.table[(int64_t)s * a.c.width + (int32_t)pos / a.c.page];
    if (id < 0 || id >= a.c.n_pages) continue;
    const int64_t to = id * a.page_bytes + ((int32_t)pos % a.c.page) * a.token_bytes;
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      const int32_t e = lane + 32 * x, h = e / a.vecs, at = (e - h * a.vecs) * 16;
      if (e < total) {
        *reinterpret_cast<uint4*>(a.K + to + h * a.head_bytes + at) = k[x];
        *reinterpret_cast<uint4*>(a.V + to + h * a.head_bytes + at) = v[x];
      }
    }
    for (int32_t e = lane + 32 * kAhead; e < total; e += 32) {
      const int32_t h = e / a.vecs, at = (e - h * a.vecs) * 16;
      const uint4 kx = *reinterpret_cast<const uint4*>(a.K_new + from + h * a.new_head_bytes + at);
      const uint4 vx = *reinterpret_cast<const uint4*>(a.V_new + from + h * a.new_head_bytes + at);
      *reinterpret_cast<uint4*>(a.K + to + h * a.head_bytes + at) = kx;
      *reinterpret_cast<uint4*>(a.V + to + h * a.head_bytes + at) = vx;
    }
  }
}

PageShape page_shape(const rocs_cache* c) {
  const int64_t es = (int64_t)elem_size(c->dtype);
  PageShape g{};
  g.K = static_cast<uint8_t*>(c->K);
  g.V = static_cast<uint8_t*>(c->V);
  g.layer_bytes = c->ld_layer * es;
  g.page_bytes = c->ld_page * es;
  g.layers = c->layers;
  int64_t n_out = c->page, ld_out = c->ld_token, n_in = c->H_kv, ld_in = c->ld_head, run = c->dh;
  if (n_out > 1 && n_in > 1 && ld_out < ld_in) {
    std::swap(n_out, n_in);
    std::swap(ld_out, ld_in);
  }
  if (n_in == 1 || ld_in == run) {
    run *= n_in;
    n_in = 1;
    if (n_out == 1 || ld_out == run) {
      run *= n_out;
      n_out = 1;
    }
  }
  g.outer = (int32_t)n_out;
  g.inner = (int32_t)n_in;
  g.outer_bytes = ld_out * es;
  g.inner_bytes = ld_in * es;
  g.vecs = (int32_t)(run * es / 16);
  return g;
}

rocs_status_t check_books(const rocs_cache* c, int32_t n, const void* workspace, size_t bytes) {
  if (!c || n < 0 || !c->refs) return ROCS_ERR_INVALID_ARG;
  if (n > kMostCounted) return ROCS_ERR_UNSUPPORTED;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || bytes < rocs_cache_workspace(c, n)) return ROCS_ERR_WORKSPACE;
  return ROCS_OK;
}

size_t claim_bytes(const rocs_cache* c) { return c->n_slots <= kBitSlots ? sizeof(uint32_t) * (size_t)((c->n_slots + 31) / 32) : 0; }

// How many CTAs copy: several rounds of the chip, so that it is busy to the end (7143 pages, two thirds in use, 6 layers: 239 us
// with 4 per SM, 229 us with 8, 215 us with 16), fewer where the pool could not give them a piece each.
unsigned copy_grid(const rocs_cache* c, const PageShape& g, int64_t most_pairs, int64_t entries) {
  const int64_t chunks = ((int64_t)g.outer * g.inner * g.vecs + kChunk - 1) / kChunk;
  const int64_t want = std::max(most_pairs * c->layers * 2 * chunks, (entries + kCopyThreads - 1) / kCopyThreads);
  return (unsigned)std::max<int64_t>(1, std::min<int64_t>(want, 16 * (int64_t)sms_of_device()));
}

}  // namespace
}  // namespace rocs

using namespace rocs;

extern "C" {

rocs_status_t rocs_cache_create(rocs_cache_t** out, rocs_dtype_t dtype, int32_t layers, int32_t n_pages, int32_t page, int32_t H_kv,
                                int32_t dh, void* K, void* V, int64_t ld_layer, int64_t ld_page, int64_t ld_token, int64_t ld_head,
                                int32_t n_slots, int32_t width, int32_t* table, int32_t* lens, int32_t* refs) {
  if (!out) return ROCS_ERR_INVALID_ARG;
  *out = nullptr;
  if ((dtype != ROCS_BF16 && dtype != ROCS_F32) || layers < 1 || n_pages < 1 || page < 1 || H_kv < 1 || dh < 1 || n_slots < 1 ||
      width < 1 || !K || !V || !table || !lens)
    return ROCS_ERR_INVALID_ARG;
  const int64_t es = (int64_t)elem_size(dtype);
  if (!aligned16(K) || !aligned16(V) || !aligned16(table) || !aligned16(lens) || !aligned16(refs) || dh * es % 16 != 0)
    return ROCS_ERR_ALIGNMENT;
  // a dimension of one entry has no stride; the others are at least a head apart
  struct Dim { int64_t n, *ld; } dims[4] = {{layers, &ld_layer}, {n_pages, &ld_page}, {page, &ld_token}, {H_kv, &ld_head}};
  for (auto& d : dims) {
    if (d.n == 1) *d.ld = 0;
    if (*d.ld * es % 16 != 0) return ROCS_ERR_ALIGNMENT;
    if (*d.ld * es >= (1ll << 40)) return ROCS_ERR_UNSUPPORTED;
  }
  // written to, so no two elements may share memory: each dimension strides over all that the closer ones span
  std::sort(dims, dims + 4, [](const auto& x, const auto& y) { return *x.ld < *y.ld; });
  int64_t span = dh;
  for (const auto& d : dims)
    if (d.n > 1) {
      if (*d.ld < span) return ROCS_ERR_INVALID_ARG;
      span += (d.n - 1) * *d.ld;
    }
  // (width: prefix sums over 1024 rows of the table stay in 32 bits; positions: so does the next multiple of a block or a page)
  if (dh > 256 || (int64_t)width * page > (1ll << 30) || width > (1 << 20) || (int64_t)page * H_kv * dh > 0x7fffffffLL ||
      n_pages > kMostCounted || n_slots > kMostCounted)
    return ROCS_ERR_UNSUPPORTED;
  rocs_cache* c = new (std::nothrow) rocs_cache{dtype, layers, n_pages, page, H_kv, dh, K, V, ld_layer, ld_page, ld_token, ld_head,
                                                n_slots, width, table, lens, refs};
  if (!c) return ROCS_ERR_INVALID_ARG;
  *out = c;
  return ROCS_OK;
}

rocs_status_t rocs_cache_destroy(rocs_cache_t* cache) {
  delete cache;
  return ROCS_OK;
}

size_t rocs_cache_workspace(const rocs_cache_t* c, int32_t n) {
  if (!c || n < 0) return 0;
  return round_up(books_words(c->n_slots, n, c->n_pages) * sizeof(int32_t), 256);
}

rocs_status_t rocs_cache_extend(const rocs_cache_t* c, const rocs_plan_t* plan, const int32_t* slots, int32_t* first, int32_t* report,
                                void* workspace, size_t bytes, void* stream_) {
  if (!plan || (plan->R > 0 && !first)) return ROCS_ERR_INVALID_ARG;
  const rocs_status_t st = check_books(c, plan->R, workspace, bytes);
  if (st != ROCS_OK) return st;
  cudaStream_t stream = (cudaStream_t)stream_;
  const Books b = books_in(workspace, c, plan->R);
  ROCS_ALLOW_SMEM(extend_kernel, kBitSlots / 8);
  const rocs_status_t launched = launch_dependent(extend_kernel, dim3(1), kBookThreads, claim_bytes(c), stream, books_of(c), slots,
                                                  plan->cand_offsets, plan->R, b, first, report);
  if (launched != ROCS_OK) return launched;
  const PageShape g = page_shape(c);
  return launch_dependent(copy_pages_kernel, dim3(copy_grid(c, g, std::min(plan->R, c->n_pages), 0)), kCopyThreads, 0, stream, g,
                          books_of(c), b, nullptr);
}

static rocs_status_t fork_or_truncate(const rocs_cache_t* c, int32_t n, const int32_t* parents, const int32_t* slots, const int32_t* keep,
                                      int32_t* report, void* workspace, size_t bytes, cudaStream_t stream) {
  const rocs_status_t st = check_books(c, n, workspace, bytes);
  if (st != ROCS_OK) return st;
  const Books b = books_in(workspace, c, n);
  const int64_t most = (int64_t)n * c->width;
  const bool one = most <= kOneCtaEntries;
  ROCS_ALLOW_SMEM(check_kernel, kBitSlots / 8);
  const rocs_status_t launched =
      launch_dependent(check_kernel, dim3(1), kBookThreads, claim_bytes(c), stream, books_of(c), parents, slots, keep, n, b, report, one);
  if (launched != ROCS_OK || one) return launched;
  return launch_dependent(apply_kernel, dim3((unsigned)std::min<int64_t>((most + 255) / 256, 4 * (int64_t)sms_of_device())), 256, 0, stream,
                          books_of(c), parents, slots, n, b);
}

rocs_status_t rocs_cache_fork(const rocs_cache_t* c, int32_t n, const int32_t* parents, const int32_t* children, int32_t* report,
                              void* workspace, size_t bytes, void* stream) {
  if (n > 0 && (!parents || !children)) return ROCS_ERR_INVALID_ARG;
  static const int32_t* const none = nullptr;
  return fork_or_truncate(c, n, parents, children, none, report, workspace, bytes, (cudaStream_t)stream);
}

rocs_status_t rocs_cache_truncate(const rocs_cache_t* c, int32_t n, const int32_t* slots, const int32_t* keep, int32_t* report,
                                  void* workspace, size_t bytes, void* stream) {
  if (n > 0 && !slots) return ROCS_ERR_INVALID_ARG;
  return fork_or_truncate(c, n, nullptr, slots, keep, report, workspace, bytes, (cudaStream_t)stream);
}

rocs_status_t rocs_cache_compact(const rocs_cache_t* c, int32_t* table_out, int32_t* refs_out, int32_t* report, void* workspace,
                                 size_t bytes, void* stream_) {
  if (!aligned16(table_out) || !aligned16(refs_out)) return ROCS_ERR_ALIGNMENT;
  const rocs_status_t st = check_books(c, 0, workspace, bytes);
  if (st != ROCS_OK) return st;
  cudaStream_t stream = (cudaStream_t)stream_;
  const Books b = books_in(workspace, c, 0);
  const rocs_status_t launched = launch_dependent(compact_kernel, dim3(1), kBookThreads, 0, stream, books_of(c), b,
                                                  refs_out ? refs_out : c->refs, report);
  if (launched != ROCS_OK) return launched;
  const PageShape g = page_shape(c);
  return launch_dependent(copy_pages_kernel, dim3(copy_grid(c, g, c->n_pages / 2, (int64_t)c->n_slots * c->width)), kCopyThreads, 0,
                          stream, g, books_of(c), b, table_out ? table_out : c->table);
}

rocs_status_t rocs_cache_append(const rocs_cache_t* c, int32_t layer, const rocs_plan_t* plan, const int32_t* slots,
                                const int32_t* first, const void* K_new, const void* V_new, int64_t ld_token, int64_t ld_head,
                                void* stream) {
  if (!c || !plan || layer < 0 || layer >= c->layers) return ROCS_ERR_INVALID_ARG;
  if (plan->N == 0) return ROCS_OK;
  if (!first || !K_new || !V_new) return ROCS_ERR_INVALID_ARG;
  const int64_t es = (int64_t)elem_size(c->dtype);
  if (!aligned16(K_new) || !aligned16(V_new) || ld_token * es % 16 != 0 || ld_head * es % 16 != 0) return ROCS_ERR_ALIGNMENT;
  if (ld_token < 0 || ld_head < 0) return ROCS_ERR_INVALID_ARG;
  AppendArgs a{};
  a.c = books_of(c);
  a.slots = slots;
  a.off = plan->cand_offsets;
  a.first = first;
  a.R = plan->R;
  a.N = plan->N;
  a.H_kv = c->H_kv;
  a.vecs = (int32_t)(c->dh * es / 16);
  a.K = static_cast<uint8_t*>(c->K) + layer * c->ld_layer * es;
  a.V = static_cast<uint8_t*>(c->V) + layer * c->ld_layer * es;
  a.page_bytes = c->ld_page * es;
  a.token_bytes = c->ld_token * es;
  a.head_bytes = c->ld_head * es;
  a.K_new = static_cast<const uint8_t*>(K_new);
  a.V_new = static_cast<const uint8_t*>(V_new);
  a.new_token_bytes = ld_token * es;
  a.new_head_bytes = ld_head * es;
  const int64_t ctas = (plan->N + 7) / 8;
  return launch_dependent(append_kernel, dim3((unsigned)std::min<int64_t>(ctas, 16 * (int64_t)sms_of_device())), 256, 0,
                          (cudaStream_t)stream, a);
}

}  // extern "C"
