// What the attention kernels over the paged cache share: parameters, the rows' visible keys, and the division of a
// launch's work.
//
// Work is counted in key blocks.  A tile is a run of a request's rows under one key head; it costs as many units as it has
// key blocks (one if it has none: zeros are written).  All tiles of the launch stand in a line, tile by tile and inside
// one block by block, and the line is cut into as many equal pieces as there are CTAs: every CTA gets the same number of
// blocks whatever the lengths, which only the device knows.  A tile that a cut goes through leaves unnormalised parts in
// the workspace, and a second small kernel joins them in the order of the keys.  At most two parts per CTA.  What a tile takes
// beside its blocks (loading Q, the last products, writing O) counts as blocks too: tiles of few keys would make some CTAs
// late.
#pragma once
#include <cuda_bf16.h>

#include "cache.h"
#include "sm100_ptx.cuh"

namespace rocs {

constexpr int kLocalEntries = 128;  // up to this many tiles (without heads) every CTA finds them itself,
constexpr int kLocalLine = 256;     // up to this many the line of tiles that a launch in front found

// A run of rows of one request: everything a kernel has to know about it but the head.
struct AttnEntry {
  int32_t slot;     // -1: none
  int32_t L;        // keys of the slot
  int32_t row0, count;  // rows of the batch
  int32_t pos0;     // where the first of them stands
  int32_t prefix;   // keys visible to all rows
  int32_t blk0, blocks;
};

struct AttnMeta {   // of a CTA whose first piece continues a tile that the CTA in front began
  AttnEntry entry;
  int32_t head;
  int32_t parts;    // of the tile; 0: no such piece
  int32_t place;    // of the first of them
  int32_t pad;
};

struct CacheAttn {
  const uint8_t *K, *V;  // of the layer
  int64_t page_bytes, token_bytes, head_bytes;
  int32_t n_pages, page, page_shift;  // page_shift < 0: not a power of two
  int32_t dh, n_slots, width;
  const int32_t *table, *lens, *slots, *off, *begin, *prefix;
  const Tile* tiles;  // null: request e is entry e
  int32_t entries, causal;
  // query heads: `group` of them per tile row, `heads` groups, `per_kv` groups per key head
  int32_t group, heads, per_kv, rows_per_tile;  // rows_per_tile: of the batch
  const uint8_t* Q;
  uint8_t* O;
  int64_t q_row_bytes, q_head_bytes, o_row_bytes, o_head_bytes;
  // scores in units of 1 / unit powers of two: scale * log2(e) / unit; capped: scale / cap, then cap * log2(e) / unit
  float scale, cap, unit;
  const float* slopes;
  int32_t block, min_shift; // keys of a block, least units of a CTA (2^)
  int32_t extra;            // units of a tile beside its blocks'
  int32_t light_rows;       // a block weighs 1 in a tile of up to so many batch rows, otherwise 2
  int32_t tile_rows;        // rows of a tile as the parts hold them (batch rows x group, rounded up)
  // workspace
  int64_t* line_global;     // [entries + 1]
  AttnEntry* entries_global;
  bool entries_made, listed;  // the entries, and the line too, were made by launches in front
  AttnMeta* meta;           // [CTAs]
  float* parts;             // [2 CTAs][tile_rows][dh], then [2 CTAs][tile_rows][2]: reference and sum
  uint32_t* status;
};

// Tensor map of the layer's K or V, [pages][heads][rows of a page][dh], for blocks of `keys` keys.
inline bool make_page_map(CUtensorMap* map, const void* base, const CacheAttn& p, int32_t H_kv, int32_t keys) {
  auto stride = [&](int64_t bytes) { return bytes > 0 ? (uint64_t)bytes : (uint64_t)p.dh * 2; };  // a single entry has none
  const uint64_t dims[4] = {(uint64_t)p.dh, (uint64_t)p.page, (uint64_t)H_kv, (uint64_t)p.n_pages};
  const uint64_t strides[3] = {stride(p.token_bytes), stride(p.head_bytes), stride(p.page_bytes)};
  const uint32_t box[4] = {p.dh == 32 ? 32u : 64u, (uint32_t)(p.page < keys ? p.page : keys), 1, 1};
  return make_tensor_map_bf16(map, base, 4, dims, strides, box);
}

#ifdef __CUDACC__
struct AttnLine {
  int64_t line[kLocalLine + 1];
  AttnEntry entry[kLocalEntries];
  uint32_t sums[kLocalLine / 32];
};
struct AttnLineView {
  const int64_t* line;
  const AttnEntry* entry;
};

// The first keys and one past the last that batch row `row0 + t` of the entry sees, and where the row stands.
struct RowKeys {
  int32_t lo, hi, pos;
};
__device__ __forceinline__ RowKeys attn_row(const CacheAttn& p, const AttnEntry& e, int32_t t) {
  RowKeys k;
  k.pos = p.causal ? e.pos0 + t : e.pos0;
  k.lo = p.begin ? max(p.begin[e.row0 + t], 0) : 0;
  k.hi = p.causal ? min(max(k.pos + 1, e.prefix), e.L) : e.L;
  return k;
}

// Entry i but for its first visible key, which takes all of its rows where rows begin somewhere.
__device__ __forceinline__ AttnEntry attn_entry(const CacheAttn& p, int32_t i) {
  AttnEntry e;
  int32_t r = i, n;
  if (p.tiles != nullptr) {
    const Tile t = p.tiles[i];
    r = t.req;
    e.row0 = t.cand0;
    e.count = t.count;
    n = p.off[r + 1] - p.off[r];
  } else {
    e.row0 = p.off[r];
    e.count = n = p.off[r + 1] - e.row0;
  }
  const int32_t s = p.slots ? p.slots[r] : r;
  e.slot = s >= 0 && s < p.n_slots ? s : -1;
  e.L = e.slot >= 0 ? min(max(p.lens[e.slot], 0), p.width * p.page) : 0;
  e.pos0 = p.causal ? e.L - n + (e.row0 - p.off[r]) : e.L;
  e.prefix = p.causal && p.prefix ? max(p.prefix[r], 0) : 0;
  return e;
}
__device__ __forceinline__ void attn_blocks(const CacheAttn& p, AttnEntry& e, int32_t first_key) {
  const int32_t last = p.causal ? min(max(e.pos0 + e.count, e.prefix), e.L) : e.L;
  e.blk0 = first_key / p.block;
  e.blocks = last > first_key ? (last + p.block - 1) / p.block - e.blk0 : 0;
}
// Units of a tile: `extra` for its beginning and end, and a block's weight for each block.
__device__ __forceinline__ int32_t attn_weight(const CacheAttn& p, const AttnEntry& e) { return e.count > p.light_rows ? 2 : 1; }
__device__ __forceinline__ uint32_t attn_cost(const CacheAttn& p, const AttnEntry& e) {
  return e.count > 0 ? (uint32_t)(p.extra + max(e.blocks, 1) * attn_weight(p, e)) : 0u;
}

// The line, found by the CTA's THREADS threads (all call this) or by the launch in front.
template <int THREADS>
__device__ __forceinline__ AttnLineView attn_line(const CacheAttn& p, AttnLine& mem) {
  if (p.listed) return AttnLineView{p.line_global, p.entries_global};
  static_assert(kLocalLine % 32 == 0 && kLocalLine <= 2 * THREADS && THREADS >= kLocalEntries, "two tiles per thread");
  const AttnEntry* entries = mem.entry;
  if (p.entries_made) {
    entries = p.entries_global;
  } else {
    if ((int32_t)threadIdx.x < p.entries) {
      AttnEntry e = attn_entry(p, threadIdx.x);
      int32_t first = 0;
      if (p.begin) {
        first = 0x7fffffff;
        for (int32_t t = 0; t < e.count; ++t) first = min(first, max(p.begin[e.row0 + t], 0));
      }
      attn_blocks(p, e, first);
      mem.entry[threadIdx.x] = e;
    }
    __syncthreads();
  }
  // (a tile's cost is below 2^26: 32 of them stay in 32 bits)
  uint32_t cost[2], incl[2];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int32_t i = threadIdx.x + r * THREADS;
    cost[r] = i < p.entries ? attn_cost(p, entries[i]) : 0u;
    incl[r] = cost[r];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t up = __shfl_up_sync(0xffffffffu, incl[r], o);
      if ((int)(threadIdx.x % 32) >= o) incl[r] += up;
    }
    if (threadIdx.x % 32 == 31 && i < kLocalLine) mem.sums[i / 32] = incl[r];
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int32_t i = threadIdx.x + r * THREADS;
    if (i < kLocalLine && i < p.entries) {
      int64_t base = 0;
      for (int w = 0; w < i / 32; ++w) base += mem.sums[w];
      mem.line[i] = base + (incl[r] - cost[r]);
      if (i == p.entries - 1) mem.line[p.entries] = base + incl[r];
    }
  }
  if (p.entries == 0 && threadIdx.x == 0) mem.line[0] = 0;
  __syncthreads();
  return AttnLineView{mem.line, entries};
}

// A CTA's way along its piece of the line.
struct AttnWalk {
  int64_t u, end;      // units
  int64_t tile_begin;  // unit at which the tile at hand begins
  int32_t entry, head, cost, weight;
  bool first;          // the piece at hand is the CTA's first
  // x / d for 0 < d < 2^31; most lines are short enough for one instruction's worth of division
  __device__ __forceinline__ static int64_t over(int64_t x, int32_t d) {
    return x >> 32 == 0 ? (int64_t)((uint32_t)x / (uint32_t)d) : x / d;
  }
  // The tile that unit x < total is in, and x moved down to where a piece may begin: the tile's first unit, or a block.  All
  // lanes of a warp call it: a line in shared memory is looked through 32 tiles at a time.
  __device__ __forceinline__ int64_t find(const CacheAttn& p, const AttnLineView& v, int64_t x) {
    const int64_t of_heads = over(x, p.heads);  // an entry begins at or before x where its line does at or before this
    int32_t lo = 0;                             // largest such entry
    if (p.listed) {
      int32_t hi = p.entries;
      while (hi - lo > 1) {
        const int32_t mid = lo + (hi - lo) / 2;
        if (v.line[mid] <= of_heads) lo = mid; else hi = mid;
      }
    } else {
      int32_t begun = 0;
      for (int32_t i0 = 0; i0 < p.entries; i0 += 32) {
        const int32_t i = i0 + (int32_t)(threadIdx.x % 32);
        begun += __popc(__ballot_sync(0xffffffffu, i < p.entries && v.line[i] <= of_heads));
      }
      lo = begun - 1;
    }
    entry = lo;
    const int64_t begin = v.line[lo];
    cost = (int32_t)(v.line[lo + 1] - begin);
    head = (int32_t)over(x - begin * p.heads, cost);
    tile_begin = begin * p.heads + (int64_t)head * cost;
    weight = attn_weight(p, v.entry[lo]);
    const int32_t block = ((int32_t)(x - tile_begin) - p.extra) >> (weight - 1);
    return block <= 0 ? tile_begin : tile_begin + p.extra + block * weight;
  }
  // false: nothing for this CTA.  Its thread NOTER, one that has little else to do, notes what the joining kernel needs.
  template <int NOTER>
  __device__ __forceinline__ bool start(const CacheAttn& p, const AttnLineView& v) {
    const int64_t total = v.line[p.entries] * p.heads;
    const int32_t ctas = (int32_t)min((int64_t)gridDim.x, max(total >> p.min_shift, (int64_t)1));
    const int32_t i = blockIdx.x;
    u = end = 0;
    first = true;
    if (i >= ctas || total == 0) {
      if (threadIdx.x == NOTER) p.meta[i].parts = 0;
      return false;
    }
    // the first `more` CTAs have a unit more than the others
    const int64_t each = over(total, ctas);
    const int32_t more = (int32_t)(total - each * ctas);
    auto cut = [&](int32_t x) { return each * x + min(x, more); };
    end = i + 1 < ctas ? find(p, v, cut(i + 1)) : total;
    u = find(p, v, cut(i));
    if (threadIdx.x == NOTER) {
      AttnMeta m;
      m.parts = 0;
      if (u > tile_begin && u < end) {
        // the CTA in front began the tile if it is cut in front of the tile's second block, and it was its first piece if it
        // is not cut in front of the tile
        const int64_t in_front = cut(i - 1), last = tile_begin + cost - 1;
        if (in_front < tile_begin + p.extra + weight) {
          m.entry = v.entry[entry];
          m.head = head;
          const int64_t longer = (each + 1) * more;  // units of the longer CTAs; the one that has unit `last`:
          const int32_t at = last < longer ? (int32_t)(last / (each + 1)) : more + (int32_t)((last - longer) / each);
          m.parts = at - (i - 1) + 1;
          m.place = 2 * (i - 1) + (in_front >= tile_begin ? 0 : 1);
        }
      }
      p.meta[i] = m;
    }
    return u < end;
  }
  __device__ __forceinline__ bool more() const { return u < end; }
  __device__ __forceinline__ int32_t block0(const CacheAttn& p) const {
    return u == tile_begin ? 0 : ((int32_t)(u - tile_begin) - p.extra) >> (weight - 1);
  }
  __device__ __forceinline__ int32_t blocks(const CacheAttn& p) const {
    return (((int32_t)(min(end, tile_begin + cost) - tile_begin) - p.extra) >> (weight - 1)) - block0(p);
  }
  __device__ __forceinline__ bool whole() const { return u == tile_begin && end >= tile_begin + cost; }
  // where a part goes: a CTA's first piece to its first place, otherwise (its last) to the second
  __device__ __forceinline__ int32_t part() const { return 2 * (int32_t)blockIdx.x + (first ? 0 : 1); }
  __device__ __forceinline__ void next(const CacheAttn& p, const AttnLineView& v) {
    tile_begin += cost;
    u = tile_begin;
    first = false;
    if (u >= end) return;
    if (++head == p.heads) {
      head = 0;
      do ++entry; while (v.line[entry + 1] == v.line[entry]);
      cost = (int32_t)(v.line[entry + 1] - v.line[entry]);
      weight = attn_weight(p, v.entry[entry]);
    }
  }
};

__device__ __forceinline__ float* attn_part(const CacheAttn& p, int32_t part) { return p.parts + (int64_t)part * p.tile_rows * p.dh; }
__device__ __forceinline__ float2* attn_part_sums(const CacheAttn& p, int32_t ctas_of_grid, int32_t part) {
  return reinterpret_cast<float2*>(p.parts + 2 * (int64_t)ctas_of_grid * p.tile_rows * p.dh) + (int64_t)part * p.tile_rows;
}

__device__ __forceinline__ int32_t page_of(const CacheAttn& p, int32_t j) { return p.page_shift >= 0 ? j >> p.page_shift : j / p.page; }

// Byte offset of key j of the slot in K or V (without the head), -1 where its page is none of the pool's.
__device__ __forceinline__ int64_t key_offset(const CacheAttn& p, int32_t slot, int32_t j) {
  const int32_t at = page_of(p, j), id = p.table[(int64_t)slot * p.width + at];
  if (id < 0 || id >= p.n_pages) return -1;
  return id * p.page_bytes + (int64_t)(j - at * p.page) * p.token_bytes;
}

__device__ __forceinline__ float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// tanh(t) as 1 - 2 / (1 + e^2t), absolute error about 1e-7 (two instructions of the special-function unit; tanh.approx is one,
// and 2^-11 off, which capped scores of 50 would show).  A score has that cap times: for caps of up to kShortCap, where it is
// 6e-6, or scores beyond 3/4 of the cap.
constexpr float kShortCap = 64.f;
__device__ __forceinline__ float tanh_far(float t) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + ex2_approx(t * 2.8853900817779268f)));
  return fmaf(-2.f, r, 1.f);
}
// tanh(t) to 1.7e-7 of its value, however small: a cap far above the scores (a caller's "none") leaves nothing of an absolute
// error.  Up to 3/4 t P(t^2), fitted for the least relative error (3e-8, 1.3e-7 with fp32's roundings).
constexpr float kTanhRange = 0.75f;
constexpr float kTanh1 = -0.3333306908607483f, kTanh2 = 0.1332651972770691f, kTanh3 = -0.053390201181173325f,
                kTanh4 = 0.01966479979455471f, kTanh5 = -0.004769410938024521f;
__device__ __forceinline__ float tanh_of(float t) {
  const float u = t * t;
  float r = fmaf(kTanh5, u, kTanh4);
  r = fmaf(r, u, kTanh3);
  r = fmaf(r, u, kTanh2);
  r = fmaf(r, u, kTanh1);
  const float near = fmaf(r, u, 1.f) * t, far = tanh_far(t);  // (both: a branch around either costs more)
  return fabsf(t) <= kTanhRange ? near : far;
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool there) {
  const int n = there ? 16 : 0;  // 0: zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __nv_bfloat162 h2 = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h2);
}

// One row over keys k0..k1-1, by one warp in fp32: reference m (log2 units), sum l, unnormalised output columns
// lane + 32 c.  For rows of the tensor-core kernels that came out non-finite: there a key that the row does not see has
// weight 0, but 0 x (NaN or Inf in its value) is not 0.  Here such keys are not looked at; what is not finite because of
// keys that the row does see comes out the same again.
template <int DH>
__device__ __forceinline__ void attn_row_by_hand(const CacheAttn& p, const AttnEntry& e, int64_t kv_head_bytes, const uint8_t* q_row,
                                                 const RowKeys& keys, float slope, int32_t k0, int32_t k1, float& m, float& l,
                                                 float (&acc)[DH / 32]) {
  const int lane = threadIdx.x % 32;
  m = -INFINITY;
  l = 0.f;
#pragma unroll
  for (int c = 0; c < DH / 32; ++c) acc[c] = 0.f;
  k0 = max(k0, keys.lo);
  k1 = min(k1, keys.hi);
  for (int32_t j0 = k0; j0 < k1; j0 += 32) {
    const int32_t j = j0 + lane;
    float x = -INFINITY;
    const int64_t off = j < k1 ? key_offset(p, e.slot, j) : -1;
    if (j < k1) {
      float s = 0.f;
      if (off >= 0) {
        const uint4* k = reinterpret_cast<const uint4*>(p.K + off + kv_head_bytes);
        const uint4* q = reinterpret_cast<const uint4*>(q_row);
#pragma unroll 1
        for (int v = 0; v < DH / 8; ++v) {
          const uint4 a = k[v], b = q[v];
          const uint32_t ka[4] = {a.x, a.y, a.z, a.w}, qb[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s = fmaf(__uint_as_float(qb[i] << 16), __uint_as_float(ka[i] << 16), s);
            s = fmaf(__uint_as_float(qb[i] & 0xffff0000u), __uint_as_float(ka[i] & 0xffff0000u), s);
          }
        }
      }
      x = s * p.scale;
      if (p.cap > 0.f) x = p.cap * tanh_of(x);
      if (p.slopes) x -= slope * fabsf((float)(keys.pos - j));
    }
    float mx = x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    const float m_new = fmaxf(m, mx), a = m == m_new ? 1.f : exp2f(m - m_new);
    const float w = x == -INFINITY ? 0.f : exp2f(x - m_new);
    l = fmaf(l, a, w);
    m = m_new;
#pragma unroll
    for (int c = 0; c < DH / 32; ++c) acc[c] *= a;
    const int32_t here = min(32, k1 - j0);
    for (int32_t k = 0; k < here; ++k) {
      const float wk = __shfl_sync(0xffffffffu, w, k);
      const int64_t at = __shfl_sync(0xffffffffu, off, k);
      if (at < 0) continue;
      const __nv_bfloat16* v = reinterpret_cast<const __nv_bfloat16*>(p.V + at + kv_head_bytes);
#pragma unroll
      for (int c = 0; c < DH / 32; ++c) acc[c] = fmaf(wk, __bfloat162float(v[lane + 32 * c]), acc[c]);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
}

__device__ __forceinline__ float slope_of(const CacheAttn& p, int32_t q_head) {
  return p.slopes ? p.slopes[q_head] * 1.4426950408889634f : 0.f;
}
#endif

// The kernels.  Each takes the launch's parameters; the grid is the number of CTAs that may share the line.
rocs_status_t attn_general(rocs_dtype_t dt, const CacheAttn& p, int32_t grid, cudaStream_t stream);
// bf16, head dimension 32, 64 or 128, on warp-level tensor cores; tiles of 16 rows (keys split over the warps) or 64.
constexpr int kMmaKeys = 64;
int attn_mma_ctas_per_sm(int32_t dh);
rocs_status_t attn_mma(const CacheAttn& p, int32_t grid, cudaStream_t stream);
// The same tiles of up to 16 rows with pages of 8, 16, 32 or a multiple of 64 rows: loads by tensor maps.
constexpr int kFewKeys = 64;
bool attn_few_supported(int32_t dh, int32_t page);
int attn_few_ctas_per_sm(int32_t dh);
rocs_status_t attn_few(const CacheAttn& p, int32_t H_kv, int32_t grid, cudaStream_t stream);
// bf16, head dimension 64 or 128, pages of 8, 16, 32, 64 or a multiple of 128 rows, on tcgen05; tiles of 256 rows.
constexpr int kUmmaKeys = 128;
bool attn_umma_supported(int32_t dh, int32_t page);
rocs_status_t attn_umma(const CacheAttn& p, int32_t H, int32_t H_kv, int64_t N, int32_t grid, cudaStream_t stream);

}  // namespace rocs
