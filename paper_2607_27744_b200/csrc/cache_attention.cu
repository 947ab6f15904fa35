// Attention over the paged cache: arguments, choice of kernel, the line of work, the joining of parts, and the general
// kernel (fp32, head dimensions that the tensor-core kernels do not take).
#include <algorithm>
#include <cmath>
#include <limits>

#include "cache_attn.cuh"

namespace rocs {
namespace {

constexpr int kLineThreads = 1024;
constexpr float kLog2e = 1.4426950408889634f;

// The tiles of a launch that has more of them than a CTA's shared memory keeps, or whose rows begin somewhere (a tile's first
// key takes a look at every row): a warp per tile.
constexpr int kEntryThreads = 256;
__global__ void __launch_bounds__(kEntryThreads) entries_kernel(CacheAttn p) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int lane = threadIdx.x % 32;
  const int32_t i = blockIdx.x * (kEntryThreads / 32) + threadIdx.x / 32;
  if (i >= p.entries) return;
  AttnEntry e = attn_entry(p, i);
  int32_t first = 0;
  if (p.begin) {
    first = 0x7fffffff;
    for (int32_t t = lane; t < e.count; t += 32) first = min(first, max(p.begin[e.row0 + t], 0));
    first = __reduce_min_sync(0xffffffffu, first);
  }
  attn_blocks(p, e, first);
  if (lane == 0) p.entries_global[i] = e;
}

// The line of more tiles than a CTA's shared memory keeps.
__global__ void __launch_bounds__(kLineThreads, 1) line_kernel(CacheAttn p) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  __shared__ uint64_t sums[kLineThreads / 32];
  uint64_t base = 0;
  for (int32_t i0 = 0; i0 < p.entries; i0 += kLineThreads) {
    const int32_t i = i0 + (int32_t)threadIdx.x;
    const uint32_t cost = i < p.entries ? attn_cost(p, p.entries_global[i]) : 0u;
    uint32_t incl = cost;  // (of 32 tiles: 32 bits)
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    if (lane == 31) sums[warp] = incl;
    __syncthreads();
    uint64_t before = base, total = 0;
    for (int w = 0; w < kLineThreads / 32; ++w) {
      if (w < warp) before += sums[w];
      total += sums[w];
    }
    if (i < p.entries) p.line_global[i] = (int64_t)(before + incl - cost);
    base += total;
    __syncthreads();
  }
  if (threadIdx.x == 0) p.line_global[p.entries] = (int64_t)base;
}

template <typename T>
__device__ __forceinline__ void store_row(uint8_t* out, int32_t c, float v) {
  if constexpr (sizeof(T) == 4) reinterpret_cast<float*>(out)[c] = v;
  else reinterpret_cast<__nv_bfloat16*>(out)[c] = __float2bfloat16_rn(v);
}

// Joins the parts of the tiles that a cut went through: O = sum_i 2^(m_i - M) O_i / sum_i 2^(m_i - M) l_i, part by part in
// the order of the keys with the largest reference so far as M.  Lanes are output columns; blockIdx.x is the cut.  A warp per
// row, or the block's four warps per row where there are more than kFewParts parts (a long sequence over the whole chip: 2
// rows of 17000 keys, 4 key heads of 64, 55 parts each, 23 us with a warp per row), each with every fourth group of four parts.
// Four parts are fetched at once: the kernel is a few trips to memory long.
constexpr int kJoinThreads = 128, kFewParts = 8;
template <int NV>
struct Joined {
  float M = -INFINITY, l = 0.f, acc[NV];
  __device__ __forceinline__ void add(float m, float sum, const float (&o)[NV], float unit) {
    // a part in which the row saw no key, or only scores of -inf, adds nothing (its sum is 0, or NaN)
    if (m == -INFINITY) {
      l += sum;
      return;
    }
    const float M_new = fmaxf(M, m), a = M == M_new ? 1.f : exp2f((M - M_new) * unit), w = exp2f((m - M_new) * unit);
    M = M_new;
    l = fmaf(l, a, w * sum);
#pragma unroll
    for (int c = 0; c < NV; ++c) acc[c] = fmaf(acc[c], a, w * o[c]);
  }
};
template <typename T, int NV>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(CacheAttn p, int32_t grid) {
  __shared__ float other[3][NV * 32 + 2];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const AttnMeta m = p.meta[blockIdx.x];
  if (m.parts == 0) return;
  const AttnEntry& e = m.entry;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  auto place = [&](int32_t i) { return i == 0 ? m.place : 2 * ((int32_t)blockIdx.x - 1 + i); };
  const bool many = m.parts > kFewParts;
  const int32_t rows = e.count * p.group, row0 = many ? blockIdx.y : blockIdx.y * 4 + warp, row_step = many ? gridDim.y : gridDim.y * 4;
  for (int32_t row = row0; row < rows; row += row_step) {
    Joined<NV> sum;
#pragma unroll
    for (int c = 0; c < NV; ++c) sum.acc[c] = 0.f;
    for (int32_t i0 = many ? warp * 4 : 0; i0 < m.parts; i0 += many ? 16 : 4) {
      float2 s[4];
      float o[4][NV];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        s[k] = make_float2(-INFINITY, 0.f);
        if (i0 + k >= m.parts) continue;
        s[k] = attn_part_sums(p, grid, place(i0 + k))[row];
        const float* from = attn_part(p, place(i0 + k)) + (int64_t)row * p.dh;
#pragma unroll
        for (int c = 0; c < NV; ++c) o[k][c] = lane + 32 * c < p.dh ? from[lane + 32 * c] : 0.f;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) sum.add(s[k].x, s[k].y, o[k], p.unit);
    }
    if (many) {  // the warps' sums, in order
      if (warp > 0) {
#pragma unroll
        for (int c = 0; c < NV; ++c) other[warp - 1][c * 32 + lane] = sum.acc[c];
        if (lane == 0) {
          other[warp - 1][NV * 32] = sum.M;
          other[warp - 1][NV * 32 + 1] = sum.l;
        }
      }
      __syncthreads();
      if (warp == 0)
        for (int w = 0; w < 3; ++w) {
          float o[NV];
#pragma unroll
          for (int c = 0; c < NV; ++c) o[c] = other[w][c * 32 + lane];
          sum.add(other[w][NV * 32], other[w][NV * 32 + 1], o, p.unit);
        }
      __syncthreads();
      if (warp > 0) continue;
    }
    const int32_t t = row / p.group;
    const RowKeys keys = attn_row(p, e, t);
    uint8_t* out = p.O + (int64_t)(e.row0 + t) * p.o_row_bytes + (m.head * p.group + row % p.group) * p.o_head_bytes;
#pragma unroll
    for (int c = 0; c < NV; ++c)
      if (lane + 32 * c < p.dh) store_row<T>(out, lane + 32 * c, keys.lo < keys.hi ? sum.acc[c] / sum.l : 0.f);
  }
}

template <typename T>
rocs_status_t join_parts(const CacheAttn& p, int32_t rows, int32_t grid, cudaStream_t stream) {
  // with as many tiles as CTAs few are cut; with fewer all are, into many parts.  (Two rounds of blocks at most: those of cuts
  // that need no joining only look that up.)
  const bool all_cut = (int64_t)p.entries * p.heads < grid;
  const int32_t most = std::max(2 * 16 * sms_of_device() / grid, 4);
  const dim3 blocks((unsigned)grid, (unsigned)std::min(all_cut ? rows : (rows + 3) / 4, most));
  if (p.dh <= 64) return launch_dependent(join_kernel<T, 2>, blocks, kJoinThreads, 0, stream, p, grid);
  if (p.dh <= 128) return launch_dependent(join_kernel<T, 4>, blocks, kJoinThreads, 0, stream, p, grid);
  return launch_dependent(join_kernel<T, 8>, blocks, kJoinThreads, 0, stream, p, grid);
}

// ---- general kernel -------------------------------------------------------------------------------
// 16 rows x blocks of 32 keys on fp32 FMAs, storage fp32 or bf16.  Queries are scaled before the product and scores stay in
// natural units up to their difference from the reference: whatever scaled score fp32 can hold is a score.  A warp has 4 rows:
// its lanes are the block's keys for the scores (one key's row of shared memory each, 4 queries broadcast) and output columns
// for P V (the probabilities broadcast).  K and V blocks are fetched with cp.async, the next while one is used.
// Long calls are bound by shared-memory reads (5 per 16 FMAs of a score, 3 per 8 of a value; 8 chunks of 200 events over 1500
// keys, 8 heads of 64: 250 us, 20 TFLOP/s), short ones by their chain: of 19 us (2 chunks over 60 keys) 9 are the launches and
// the line of work, 3.5 a piece's beginning and end, 3 a block.  Two output columns in one read were slower (305 us).
constexpr int kGenThreads = 128, kGenRows = 16, kGenKeys = 32;

template <typename T>
__host__ __device__ constexpr int gen_row_bytes(int dh) { return dh * (int)sizeof(T) + 16; }  // a row's 16-byte vectors fall on other banks than the next one's
template <typename T>
constexpr int gen_smem(int dh) { return kGenRows * dh * 4 + 4 * kGenKeys * gen_row_bytes<T>(dh); }

template <typename T>
__device__ __forceinline__ void unpack_vec(const uint4& raw, float (&v)[16 / sizeof(T)]) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    if constexpr (sizeof(T) == 4) {
      v[x] = __uint_as_float(w[x]);
    } else {
      v[2 * x] = __uint_as_float(w[x] << 16);
      v[2 * x + 1] = __uint_as_float(w[x] & 0xffff0000u);
    }
  }
}

template <typename T, int NV>
__global__ void __launch_bounds__(kGenThreads) general_kernel(const CacheAttn p) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ AttnLine line_mem;
  __shared__ __align__(16) float probs[kGenThreads / 32][kGenKeys][4];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const AttnLineView view = attn_line<kGenThreads>(p, line_mem);
  AttnWalk walk;
  if (!walk.start<kGenThreads - 1>(p, view)) return;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int32_t dh = p.dh, row_bytes = gen_row_bytes<T>(dh), vecs = dh * (int)sizeof(T) / 16;
  float* qs = reinterpret_cast<float*>(smem);
  uint8_t* kv = smem + kGenRows * dh * 4;  // [2 stages][K, V][32 keys]
  const uint32_t kv_addr = ptx::smem_u32(kv);
  const int32_t block_bytes = kGenKeys * row_bytes;
  // the vectors of a block that a thread loads: kGenThreads after one another
  const int32_t load_row = threadIdx.x / vecs, load_vec = threadIdx.x - load_row * vecs;
  const int32_t row_step = kGenThreads / vecs, vec_step = kGenThreads - row_step * vecs;

  for (; walk.more(); walk.next(p, view)) {
    const AttnEntry e = view.entry[walk.entry];
    const int32_t kv_head = walk.head / p.per_kv;
    const int64_t kv_head_bytes = kv_head * p.head_bytes;
    const int32_t rows = e.count * p.group;
    __syncthreads();  // the piece in front is done with shared memory
    // (all of a thread's vectors are asked for before the first is stored: a trip to memory each would be most of a short piece)
    constexpr int kPer = 16 / (int)sizeof(T), kQVecs = (NV * (int)sizeof(T) + 3) / 4;
    uint4 raw_q[kQVecs];
#pragma unroll
    for (int i = 0; i < kQVecs; ++i) {
      const int32_t x = threadIdx.x + i * kGenThreads, row = x / vecs;
      raw_q[i] = make_uint4(0u, 0u, 0u, 0u);
      if (row < min(rows, kGenRows))
        raw_q[i] = *reinterpret_cast<const uint4*>(p.Q + (int64_t)(e.row0 + row / p.group) * p.q_row_bytes +
                                                   (walk.head * p.group + row % p.group) * p.q_head_bytes + (x - row * vecs) * 16);
    }
#pragma unroll
    for (int i = 0; i < kQVecs; ++i) {
      const int32_t x = threadIdx.x + i * kGenThreads;
      if (x >= kGenRows * vecs) continue;
      float q[kPer];
      unpack_vec<T>(raw_q[i], q);
#pragma unroll
      for (int c = 0; c < kPer; c += 4)
        *reinterpret_cast<float4*>(qs + x * kPer + c) = make_float4(q[c] * p.scale, q[c + 1] * p.scale, q[c + 2] * p.scale, q[c + 3] * p.scale);
    }
    RowKeys keys[4];
    float slope[4], m[4], l[4], acc[4][NV];
    int32_t lo_most = 0, hi_least = 0x7fffffff;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int32_t row = warp * 4 + i;
      keys[i] = RowKeys{0, 0, 0};
      slope[i] = 0.f;
      if (row < rows) {
        keys[i] = attn_row(p, e, row / p.group);
        slope[i] = p.slopes ? p.slopes[walk.head * p.group + row % p.group] : 0.f;
      }
      lo_most = max(lo_most, keys[i].lo);
      hi_least = min(hi_least, keys[i].hi);
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int c = 0; c < NV; ++c) acc[i][c] = 0.f;
    }
    const int32_t blk0 = e.blk0 + walk.block0(p), blocks = e.blocks > 0 ? walk.blocks(p) : 0;
    const int32_t last_key = min(e.L, p.causal ? max(e.pos0 + e.count, e.prefix) : e.L);  // one past the last that any row sees
    // A lane looks up a key of the next block to load, a block ahead: a trip to memory in front of another.
    auto look_up = [&](int32_t b) {
      const int32_t j = (blk0 + b) * kGenKeys + lane;
      return b < blocks && j < last_key ? key_offset(p, e.slot, j) : -1;
    };
    int64_t ahead = look_up(0);
    auto load = [&](int32_t b) {
      const uint32_t dst = kv_addr + (b & 1) * 2 * block_bytes;
#pragma unroll 4
      for (int32_t row = load_row, v = load_vec; row < kGenKeys;) {  // (a multiple of 32 of them: whole warps)
        const int64_t at = __shfl_sync(0xffffffffu, ahead, row);
        const int64_t off = at >= 0 ? at + kv_head_bytes + v * 16 : 0;
        cp_async16(dst + row * row_bytes + v * 16, p.K + off, at >= 0);
        cp_async16(dst + block_bytes + row * row_bytes + v * 16, p.V + off, at >= 0);
        row += row_step;
        v += vec_step;
        if (v >= vecs) {
          v -= vecs;
          ++row;
        }
      }
      cp_async_commit();
      ahead = look_up(b + 1);
    };
    if (blocks > 0) load(0);
    for (int32_t b = 0; b < blocks; ++b) {
      if (b + 1 < blocks) {
        load(b + 1);
        cp_async_wait<1>();
      } else {
        cp_async_wait<0>();
      }
      __syncthreads();
      const uint8_t* kb = kv + (b & 1) * 2 * block_bytes;
      const uint8_t* vb = kb + block_bytes;
      const int32_t j0 = (blk0 + b) * kGenKeys, j = j0 + lane;
      const bool full = j0 >= lo_most && j0 + kGenKeys <= hi_least;
      float s[4] = {0.f, 0.f, 0.f, 0.f};
      const float* q = qs + warp * 4 * dh;
      const uint8_t* kr = kb + lane * row_bytes;
#pragma unroll 4
      for (int32_t v = 0; v < vecs; ++v) {
        const uint4 raw = *reinterpret_cast<const uint4*>(kr + v * 16);
        float k[kPer];
        unpack_vec<T>(raw, k);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int x = 0; x < kPer; x += 4) {
            const float4 qv = *reinterpret_cast<const float4*>(q + i * dh + v * kPer + x);
            s[i] = fmaf(qv.x, k[x], s[i]);
            s[i] = fmaf(qv.y, k[x + 1], s[i]);
            s[i] = fmaf(qv.z, k[x + 2], s[i]);
            s[i] = fmaf(qv.w, k[x + 3], s[i]);
          }
      }
      float pr[4];
      bool moves = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x = s[i];
        if (p.cap > 0.f) x = p.cap * tanhf(x);
        if (p.slopes) x -= slope[i] * fabsf((float)(keys[i].pos - j));
        if (!full && (j < keys[i].lo || j >= keys[i].hi)) x = -INFINITY;
        s[i] = x;
        moves |= x > m[i] + 8.f;  // (from -inf: any score)
      }
      // a row's reference moves where a score passes it by e^8, which fp32 sums have room for
      if (__any_sync(0xffffffffu, moves)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float mx = s[i];
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
          if (mx > m[i] + 8.f) {  // a row's own decision
            const float a = exp2f((m[i] - mx) * kLog2e);
            m[i] = mx;
            l[i] *= a;
#pragma unroll
            for (int c = 0; c < NV; ++c) acc[i][c] *= a;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        pr[i] = s[i] == -INFINITY ? 0.f : exp2f((s[i] - m[i]) * kLog2e);
        l[i] += pr[i];
      }
      // a key that a row does not see adds nothing, whatever its value holds; one that it sees does, whatever its weight
      if (!full) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (j < keys[i].lo || j >= keys[i].hi) pr[i] = -1.f;
      }
      *reinterpret_cast<float4*>(probs[warp][lane]) = make_float4(pr[0], pr[1], pr[2], pr[3]);
      __syncwarp();
      auto add_values = [&](bool masked) {
#pragma unroll 4
        for (int k = 0; k < kGenKeys; ++k) {
          const float4 w = *reinterpret_cast<const float4*>(probs[warp][k]);
          const uint8_t* vr = vb + k * row_bytes;
#pragma unroll
          for (int c = 0; c < NV; ++c) {
            const int32_t d = lane + 32 * c;
            if (d >= dh) continue;
            float x;
            if constexpr (sizeof(T) == 4) x = reinterpret_cast<const float*>(vr)[d];
            else x = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(vr)[d]);
            if (!masked || !(w.x < 0.f)) acc[0][c] = fmaf(w.x, x, acc[0][c]);
            if (!masked || !(w.y < 0.f)) acc[1][c] = fmaf(w.y, x, acc[1][c]);
            if (!masked || !(w.z < 0.f)) acc[2][c] = fmaf(w.z, x, acc[2][c]);
            if (!masked || !(w.w < 0.f)) acc[3][c] = fmaf(w.w, x, acc[3][c]);
          }
        }
      };
      if (full) add_values(false); else add_values(true);
      __syncthreads();  // the block's place may be loaded into
    }
    const bool whole = walk.whole();
    const int32_t part = walk.part();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int32_t row = warp * 4 + i;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], o);
      if (row >= rows) continue;
      if (whole) {
        uint8_t* out = p.O + (int64_t)(e.row0 + row / p.group) * p.o_row_bytes + (walk.head * p.group + row % p.group) * p.o_head_bytes;
#pragma unroll
        for (int c = 0; c < NV; ++c)
          if (lane + 32 * c < dh) store_row<T>(out, lane + 32 * c, keys[i].lo < keys[i].hi ? acc[i][c] / l[i] : 0.f);
      } else {
        float* o = attn_part(p, part) + (int64_t)row * dh;
#pragma unroll
        for (int c = 0; c < NV; ++c)
          if (lane + 32 * c < dh) o[lane + 32 * c] = acc[i][c];
        if (lane == 0) attn_part_sums(p, gridDim.x, part)[row] = make_float2(m[i], l[i]);
      }
    }
  }
}

template <typename T, int NV>
rocs_status_t launch_general(const CacheAttn& p, int32_t grid, cudaStream_t stream) {
  auto kernel = general_kernel<T, NV>;
  ROCS_ALLOW_SMEM(kernel, gen_smem<T>(32 * NV));
  return launch_dependent(kernel, dim3((unsigned)grid), kGenThreads, (size_t)gen_smem<T>(p.dh), stream, p);
}
template <typename T>
rocs_status_t general_of(const CacheAttn& p, int32_t grid, cudaStream_t stream) {
  if (p.dh <= 32) return launch_general<T, 1>(p, grid, stream);
  if (p.dh <= 64) return launch_general<T, 2>(p, grid, stream);
  if (p.dh <= 128) return launch_general<T, 4>(p, grid, stream);
  return launch_general<T, 8>(p, grid, stream);
}

enum class Kind { kGeneral, kMma, kFew, kUmma };

// Which kernel a call takes, and how its work is cut.  q_spread: neither the rows nor the heads of Q are one broadcast.
struct Choice {
  Kind kind;
  int32_t group, per_kv, heads;  // query heads per tile row, such groups per key head, groups in all
  int32_t rows_per_tile, tile_rows, block, min_shift, extra, grid;
  int64_t entries;
  bool by_request;  // no request has more than one tile
};
Choice choose(const rocs_cache* c, const rocs_plan* plan, int32_t H, int path, bool q_spread) {
  Choice x{};
  const int32_t g = H / c->H_kv, sms = sms_of_device();
  int32_t most = 16;
  x.kind = Kind::kGeneral;
  x.block = kGenKeys;
  x.min_shift = 1;
  x.extra = 1;
  if (c->dtype == ROCS_BF16 && path == ROCS_PATH_AUTO && (c->dh == 32 || c->dh == 64 || c->dh == 128)) {
    x.kind = Kind::kMma;
    x.block = kMmaKeys;
    if ((int64_t)plan->largest * g > 16) most = 64;
    else if (attn_few_supported(c->dh, c->page)) {
      x.kind = Kind::kFew;
      x.block = kFewKeys;
      x.extra = 4;
      x.min_shift = 2;
      if ((int64_t)plan->largest * g <= 8) most = 8;
    }
    // Few rows: a tile of the tcgen05 kernel takes about 6 us beside its keys, one of the other kernel 2 us and longer for each
    // key.  Rows of each of 6 requests over 250 keys, 4 heads of 64, tcgen05 and the other: 20 / 40 / 64 / 100 / 148 rows 18.0 /
    // 18.8 / 20.2 / 21.8 / 20.0 and 12.2 / 14.2 / 17.2 / 18.6 / 18.7 us; 24 requests over 1000 keys, 8 heads of 64: 40 / 64 / 100
    // rows 28.3 / 28.7 / 29.8 and 28.7 / 32.3 / 47.9; 8 over 2000, 8 heads of 128: 40 / 64 / 100 rows 26.9 / 27.9 / 30.2 and 34.8 /
    // 37.6 / 58.8.  How many keys there are is known on the device only; the table's width says how many there may be.
    // A batch of a chunk and single events goes the chunk's way, all of it: 300 rows over 4000 keys beside 48 events over 500-8000,
    // 8 heads of 64, 77 us, and 99 us as a call for the chunk (35) and one for the events (65); 8 x 4 heads of 128 130 and 154 us;
    // 40 rows beside 64 events, 8 heads of 64, 99 and 113 us.
    const bool many_keys = (int64_t)c->width * c->page >= 512;
    // (its tensor map of Q takes no stride of 0)
    if (q_spread && (int64_t)plan->largest * g > (many_keys ? 32 : 128) && attn_umma_supported(c->dh, c->page)) {
      x.kind = Kind::kUmma;
      x.block = kUmmaKeys;
      x.min_shift = 2;
      x.extra = 4;
      most = 128;  // of a side
    }
  }
  // the CTAs of one round of the chip: 128 registers a thread, and shared memory (with the line and the probabilities)
  const int smem = (c->dtype == ROCS_BF16 ? gen_smem<__nv_bfloat16>(c->dh) : gen_smem<float>(c->dh)) + (int)sizeof(AttnLine) + 4096;
  x.grid = sms * (x.kind == Kind::kUmma ? 1 : x.kind == Kind::kFew ? attn_few_ctas_per_sm(c->dh) : x.kind == Kind::kMma ? attn_mma_ctas_per_sm(c->dh) : std::min(4, 228 * 1024 / smem));
  x.group = 1;  // the largest part of the heads of a key head that fits a tile
  for (int32_t d = std::min(g, most); d >= 1; --d)
    if (g % d == 0) { x.group = d; break; }
  x.per_kv = g / x.group;
  x.heads = H / x.group;
  const int32_t sides = x.kind == Kind::kUmma ? 2 : 1;
  x.rows_per_tile = sides * (most / x.group);
  x.tile_rows = sides * most;
  x.by_request = plan->largest <= x.rows_per_tile;
  x.entries = x.by_request ? plan->R : plan_entries(plan, x.rows_per_tile);
  return x;
}

struct Places {
  size_t meta, line, entries, parts, bytes;
};
Places places(const Choice& x, int32_t dh) {
  Places w;
  w.meta = 0;
  w.line = w.meta + round_up(sizeof(AttnMeta) * (size_t)x.grid, 256);
  w.entries = w.line + round_up(sizeof(int64_t) * ((size_t)x.entries + 1), 256);
  w.parts = w.entries + round_up(sizeof(AttnEntry) * (size_t)x.entries, 256);
  w.bytes = w.parts + round_up(2 * (size_t)x.grid * x.tile_rows * ((size_t)dh + 2) * sizeof(float), 256);
  return w;
}

bool strides_ok(int64_t ld_row, int64_t ld_head, int64_t es) {
  return ld_row >= 0 && ld_head >= 0 && ld_row * es % 16 == 0 && ld_head * es % 16 == 0;
}

// Whether rows of O share memory: the larger of the two strides has to span all that the smaller one does.
bool shares_memory(int64_t rows, int64_t ld_row, int64_t heads, int64_t ld_head, int64_t dh) {
  if (rows > 1 && heads > 1)
    return ld_row < ld_head ? ld_row < dh || (ld_head - dh) / ld_row < rows - 1 : ld_head < dh || (ld_row - dh) / ld_head < heads - 1;
  return (heads > 1 && ld_head < dh) || (rows > 1 && ld_row < dh);
}

}  // namespace

rocs_status_t attn_general(rocs_dtype_t dt, const CacheAttn& p, int32_t grid, cudaStream_t stream) {
  return dt == ROCS_BF16 ? general_of<__nv_bfloat16>(p, grid, stream) : general_of<float>(p, grid, stream);
}

}  // namespace rocs

using namespace rocs;

extern "C" {

size_t rocs_cache_attention_workspace(const rocs_cache_t* c, const rocs_plan_t* plan, int32_t H) {
  if (!c || !plan || H < 1 || H % c->H_kv != 0) return 0;
  size_t most = 0;  // whichever path is in force when it is used, and whatever strides Q has
  for (int path : {ROCS_PATH_AUTO, ROCS_PATH_GENERAL})
    for (bool q_spread : {false, true}) most = std::max(most, places(choose(c, plan, H, path, q_spread), c->dh).bytes);
  return most;
}

rocs_status_t rocs_cache_attention(const rocs_cache_t* c, int32_t layer, const rocs_plan_t* plan, const int32_t* slots, int32_t H,
                                   const void* Q, int64_t ld_qt, int64_t ld_qh, int32_t causal, float scale, float cap,
                                   const float* slopes, const int32_t* begin, const int32_t* prefix, void* O, int64_t ld_ot,
                                   int64_t ld_oh, void* workspace, size_t bytes, void* stream_) {
  if (!c || !plan || layer < 0 || layer >= c->layers || H < 1 || H % c->H_kv != 0) return ROCS_ERR_INVALID_ARG;
  if ((!causal && prefix) || !(cap >= 0.f) || std::isinf(cap) || !std::isfinite(scale)) return ROCS_ERR_INVALID_ARG;
  if (plan->N == 0) return ROCS_OK;
  if (!Q || !O) return ROCS_ERR_INVALID_ARG;
  const int64_t es = (int64_t)elem_size(c->dtype);
  if (!aligned16(Q) || !aligned16(O) || !strides_ok(ld_qt, ld_qh, es) || !strides_ok(ld_ot, ld_oh, es)) return ROCS_ERR_ALIGNMENT;
  if (shares_memory(plan->N, ld_ot, H, ld_oh, c->dh)) return ROCS_ERR_INVALID_ARG;
  if (H > 65535) return ROCS_ERR_UNSUPPORTED;
  if (!(scale > 0.f)) scale = 1.0f / sqrtf((float)c->dh);
  if (!std::isfinite(scale * kLog2e) || (cap > 0.f && !std::isfinite(scale / cap))) return ROCS_ERR_INVALID_ARG;
  if (cap > 0.f && scale / cap < std::numeric_limits<float>::min()) {
    // The kernels' factor would lose bits, or be 0.  Products of fp32 stay below 2^128, so that no score is above 4 caps.  One
    // below 2^-12 of the cap is, to 2^-25 of it, what it is without a cap; if the cap is 2^64 at least, others are 2^28 apart, or
    // equal, in fp32, and under the cap still 2^18: the largest has all the weight either way.
    if (cap < 0x1p64f) return ROCS_ERR_INVALID_ARG;
    cap = 0.f;
  }
  if (!std::isfinite(cap * kLog2e)) return ROCS_ERR_INVALID_ARG;
  const Choice x = choose(c, plan, H, kernel_path(), (H == 1 || ld_qh > 0) && (plan->N == 1 || ld_qt > 0));
  const Places w = places(x, c->dh);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || bytes < w.bytes) return ROCS_ERR_WORKSPACE;
  if (x.entries > kMostCounted) return ROCS_ERR_UNSUPPORTED;
  cudaStream_t stream = (cudaStream_t)stream_;
  CacheAttn p{};
  p.K = static_cast<const uint8_t*>(c->K) + layer * c->ld_layer * es;
  p.V = static_cast<const uint8_t*>(c->V) + layer * c->ld_layer * es;
  p.page_bytes = c->ld_page * es;
  p.token_bytes = c->ld_token * es;
  p.head_bytes = c->ld_head * es;
  p.n_pages = c->n_pages;
  p.page = c->page;
  p.page_shift = -1;
  for (int s = 0; s < 31; ++s)
    if (c->page == (1 << s)) p.page_shift = s;
  p.dh = c->dh;
  p.n_slots = c->n_slots;
  p.width = c->width;
  p.table = c->table;
  p.lens = c->lens;
  p.slots = slots;
  p.off = plan->cand_offsets;
  p.begin = begin;
  p.prefix = prefix;
  p.entries = (int32_t)x.entries;
  p.causal = causal != 0;
  p.group = x.group;
  p.heads = x.heads;
  p.per_kv = x.per_kv;
  p.rows_per_tile = x.rows_per_tile;
  p.Q = static_cast<const uint8_t*>(Q);
  p.O = static_cast<uint8_t*>(O);
  p.q_row_bytes = ld_qt * es;
  p.q_head_bytes = ld_qh * es;
  p.o_row_bytes = ld_ot * es;
  p.o_head_bytes = ld_oh * es;
  p.unit = x.kind == Kind::kGeneral ? kLog2e : 1.f;
  const float to_unit = x.kind == Kind::kGeneral ? 1.f : kLog2e;
  p.scale = cap > 0.f ? scale / cap : scale * to_unit;
  p.cap = cap * to_unit;
  p.slopes = slopes;
  p.block = x.block;
  p.min_shift = x.min_shift;
  p.extra = x.extra;
  p.light_rows = x.kind == Kind::kUmma ? x.rows_per_tile / 2 : x.rows_per_tile;
  p.tile_rows = x.tile_rows;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  p.meta = reinterpret_cast<AttnMeta*>(ws + w.meta);
  p.line_global = reinterpret_cast<int64_t*>(ws + w.line);
  p.entries_global = reinterpret_cast<AttnEntry*>(ws + w.entries);
  p.parts = reinterpret_cast<float*>(ws + w.parts);
  p.status = device_status_word();
  if (!p.status) return ROCS_ERR_CUDA;
  if (!x.by_request) {
    TileList tiles;
    const rocs_status_t st = plan_tiles(plan, x.rows_per_tile, stream, &tiles);
    if (st != ROCS_OK) return st;
    p.tiles = tiles.dev;
  }
  p.listed = x.entries > kLocalLine;
  p.entries_made = x.entries > kLocalEntries || (begin && x.rows_per_tile > 8);
  if (p.entries_made) {
    const int64_t ctas = (x.entries + kEntryThreads / 32 - 1) / (kEntryThreads / 32);
    const rocs_status_t st = launch_dependent(entries_kernel, dim3((unsigned)ctas), kEntryThreads, 0, stream, p);
    if (st != ROCS_OK) return st;
  }
  if (p.listed) {
    const rocs_status_t st = launch_dependent(line_kernel, dim3(1), kLineThreads, 0, stream, p);
    if (st != ROCS_OK) return st;
  }
  const rocs_status_t st = x.kind == Kind::kUmma  ? attn_umma(p, H, c->H_kv, plan->N, x.grid, stream)
                           : x.kind == Kind::kFew ? attn_few(p, c->H_kv, x.grid, stream)
                           : x.kind == Kind::kMma ? attn_mma(p, x.grid, stream)
                                                  : attn_general(c->dtype, p, x.grid, stream);
  if (st != ROCS_OK) return st;
  const int32_t rows = (int32_t)std::min<int64_t>(x.tile_rows, (int64_t)plan->largest * x.group);  // most of a tile
  return c->dtype == ROCS_BF16 ? join_parts<__nv_bfloat16>(p, rows, x.grid, stream) : join_parts<float>(p, rows, x.grid, stream);
}

}  // extern "C"
