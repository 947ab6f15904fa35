// Attention over the paged cache on warp-level tensor cores (mma.sync m16n8k16, bf16): tiles of few rows, where the time is
// the reading of K and V.
//
// Tiles of 16 rows (a single event, or a few, of the query heads that share a key head): the 4 warps split the 64 keys of a
// block, each with a reference and sums of its own, and add up at the end of the piece.  Tiles of 64 rows (chunks of up to
// that many; page sizes and head dimensions that the tcgen05 kernel does not take): a warp has 16 of the rows and all keys
// of a block.  Either way the CTA's next blocks are in flight (cp.async, 16 bytes per thread and row, so that a page may
// have any size and rows any stride; the loads run ahead over the end of a tile into the next), and the page ids of the
// block after those are already in registers: a lookup in the table is a trip to memory in front of another.
//
// Softmax in log2 units against a reference per row that only moves when a score passes it by 2^8: most blocks then leave
// the accumulators alone, and probabilities stay below 256 (bf16 keeps its 8 bits there; their sum is taken from the
// unrounded fp32 values).
#include "cache_attn.cuh"

namespace rocs {
namespace {

constexpr int kMmaThreads = 128;

template <int DH>
struct MmaCfg {
  static constexpr int kStages = DH == 128 ? 3 : 4;
  static constexpr int kTileBytes = kMmaKeys * DH * 2;          // K or V of a block
  static constexpr int kStageBytes = 2 * kTileBytes;
  static constexpr int kMergeBytes = 16 * DH * 4 + 4 * 16 * 8;  // one warp's output, all warps' references and sums
  static constexpr int kSmem = kStages * kStageBytes + kMergeBytes;
  static constexpr int kPerSm = DH == 128 ? 2 : DH == 64 ? 3 : 4;
  static_assert(kPerSm * (kSmem + (int)sizeof(AttnLine) + 1024) <= 228 * 1024, "shared memory of an SM");
  static constexpr int kChunks = DH / 8;                        // 16-byte vectors of a row
  static constexpr int kRowsPerPass = kMmaThreads / kChunks;
  static constexpr int kPasses = kMmaKeys / kRowsPerPass;       // rows of a block that a thread loads
  // place of a row's vector: the 8 rows that one matrix load takes fall on different banks
  __device__ static uint32_t at(uint32_t row, uint32_t chunk) {
    return row * (DH * 2) + ((DH == 32 ? chunk ^ ((row >> 1) & 3) : chunk ^ (row & 7)) << 4);
  }
};

__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// MW warps along the rows, 4 / MW along the keys.
template <int DH, int MW>
__global__ void __launch_bounds__(kMmaThreads, MmaCfg<DH>::kPerSm) mma_kernel(const CacheAttn p) {
  using C = MmaCfg<DH>;
  constexpr int KW = 4 / MW, kGroups = kMmaKeys / 16 / KW;  // groups of 16 keys of a block that a warp takes
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ AttnLine line_mem;
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const AttnLineView view = attn_line<kMmaThreads>(p, line_mem);
  AttnWalk walk;
  if (!walk.start<kMmaThreads - 1>(p, view)) return;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const uint32_t sb = ptx::smem_u32(smem);
  float* merge = reinterpret_cast<float*>(smem + C::kStages * C::kStageBytes);
  float2* merge_sums = reinterpret_cast<float2*>(merge + 16 * DH);  // [4 warps][16 rows]

  // ---- loads: a way of their own along the line, ahead of the computation
  const int load_chunk = threadIdx.x % C::kChunks, load_row = threadIdx.x / C::kChunks;
  AttnWalk ahead = walk;
  int32_t ahead_b = 0, ahead_n = 0, ahead_slot = 0, ahead_blk0 = 0, ahead_last = 0;
  int64_t ahead_head = 0;
  int32_t ids[C::kPasses];  // page of the thread's rows of the next block to load, -1: none
  bool ahead_more = true;
  auto ahead_piece = [&]() {  // the piece at hand of `ahead`; pieces without keys are passed over
    while (ahead.more()) {
      const AttnEntry& e = view.entry[ahead.entry];
      if (e.blocks > 0) {
        ahead_b = 0;
        ahead_n = ahead.blocks(p);
        ahead_slot = e.slot;
        ahead_blk0 = e.blk0 + ahead.block0(p);
        ahead_last = min(e.L, p.causal ? max(e.pos0 + e.count, e.prefix) : e.L);
        ahead_head = (int64_t)(ahead.head / p.per_kv) * p.head_bytes + load_chunk * 16;
        return;
      }
      ahead.next(p, view);
    }
    ahead_more = false;
  };
  auto look_up = [&]() {
    if (!ahead_more) return;
    const int32_t* row = p.table + (int64_t)ahead_slot * p.width;
#pragma unroll
    for (int i = 0; i < C::kPasses; ++i) {
      const int32_t j = (ahead_blk0 + ahead_b) * kMmaKeys + load_row + i * C::kRowsPerPass;
      ids[i] = j < ahead_last ? row[page_of(p, j)] : -1;
    }
  };
  uint32_t load_stage = 0;
  auto load = [&]() {
    if (ahead_more) {
      const uint32_t k_dst = sb + load_stage * C::kStageBytes;
#pragma unroll
      for (int i = 0; i < C::kPasses; ++i) {
        const int32_t r = load_row + i * C::kRowsPerPass, j = (ahead_blk0 + ahead_b) * kMmaKeys + r, id = ids[i];
        const bool there = id >= 0 && id < p.n_pages;
        const int64_t off = there ? id * p.page_bytes + (int64_t)(j - page_of(p, j) * p.page) * p.token_bytes + ahead_head : 0;
        cp_async16(k_dst + C::at(r, load_chunk), p.K + off, there);
        cp_async16(k_dst + C::kTileBytes + C::at(r, load_chunk), p.V + off, there);
      }
      load_stage = load_stage + 1 == C::kStages ? 0 : load_stage + 1;
      if (++ahead_b == ahead_n) {
        ahead.next(p, view);
        ahead_piece();
      }
    }
    cp_async_commit();
    look_up();
  };
  ahead_piece();
  look_up();
#pragma unroll
  for (int s = 0; s < C::kStages - 1; ++s) load();
  uint32_t stage = 0;

  for (; walk.more(); walk.next(p, view)) {
    const AttnEntry e = view.entry[walk.entry];
    const int32_t rows = e.count * p.group;
    const int32_t row_lo = (MW == 1 ? 0 : warp * 16) + lane / 4;  // this thread's rows: row_lo and row_lo + 8
    uint32_t q[DH / 16][4];
    RowKeys keys[2];
    float slope[2], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int32_t row = row_lo + 8 * i;
      keys[i] = RowKeys{0, 0x7fffffff, 0};  // a row that does not exist asks for no mask
      slope[i] = 0.f;
      const bool there = row < rows;
      const uint8_t* src = p.Q;
      if (there) {
        keys[i] = attn_row(p, e, row / p.group);
        slope[i] = slope_of(p, walk.head * p.group + row % p.group);
        src += (int64_t)(e.row0 + row / p.group) * p.q_row_bytes + (walk.head * p.group + row % p.group) * p.q_head_bytes;
      }
#pragma unroll
      for (int k = 0; k < DH / 16; ++k)
#pragma unroll
        for (int c = 0; c < 2; ++c)
          q[k][i + 2 * c] = there ? *reinterpret_cast<const uint32_t*>(src + (k * 16 + c * 8 + 2 * (lane % 4)) * 2) : 0u;
    }
    const int32_t lo_most = __reduce_max_sync(0xffffffffu, max(keys[0].lo, keys[1].lo));
    const int32_t hi_least = __reduce_min_sync(0xffffffffu, min(keys[0].hi, keys[1].hi));
    float o[DH / 8][4];
#pragma unroll
    for (int n = 0; n < DH / 8; ++n)
#pragma unroll
      for (int c = 0; c < 4; ++c) o[n][c] = 0.f;
    const int32_t blk0 = e.blk0 + walk.block0(p), blocks = e.blocks > 0 ? walk.blocks(p) : 0;
    for (int32_t b = 0; b < blocks; ++b) {
      cp_async_wait<C::kStages - 2>();
      __syncthreads();  // the block is there for all, and all are done with the one whose place the next load takes
      load();
      const uint32_t k_tile = sb + stage * C::kStageBytes, v_tile = k_tile + C::kTileBytes;
      stage = stage + 1 == C::kStages ? 0 : stage + 1;
      const int32_t j0 = (blk0 + b) * kMmaKeys, g0 = MW == 1 ? warp * kGroups : 0;
      float s[kGroups][2][4];
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) s[g][n][c] = 0.f;
#pragma unroll
        for (int k = 0; k < DH / 16; ++k) {
          uint32_t f[4];
          ldmatrix_x4(k_tile + C::at((g0 + g) * 16 + (lane / 16) * 8 + lane % 8, 2 * k + (lane / 8) % 2), f);
          mma_bf16(s[g][0], q[k], f[0], f[1]);
          mma_bf16(s[g][1], q[k], f[2], f[3]);
        }
      }
      const bool full = j0 >= lo_most && j0 + kMmaKeys <= hi_least;
      float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) s[g][n][c] *= p.scale;
      if (p.cap > 0.f) {  // (24 chunks of 8-120 rows, 8 heads of 32: 33.2 us, 35.5 us with tanh_of for all caps)
        const bool far = p.cap <= kShortCap;  // (in log2 units, two thirds of it in the caller's)
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int c = 0; c < 4; ++c) s[g][n][c] = p.cap * (far ? tanh_far(s[g][n][c]) : tanh_of(s[g][n][c]));
      }
      if (p.slopes || !full) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g)
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const int32_t j = j0 + (g0 + g) * 16 + n * 8 + 2 * (lane % 4) + c % 2;
              const RowKeys& rk = keys[c / 2];
              float x = s[g][n][c];
              if (p.slopes) x -= slope[c / 2] * fabsf((float)(rk.pos - j));
              s[g][n][c] = j < rk.lo || j >= rk.hi ? -INFINITY : x;
            }
      }
#pragma unroll
      for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) mx[c / 2] = fmaxf(mx[c / 2], s[g][n][c]);
      bool moves = false;
      float m_new[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 1));
        mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 2));
        m_new[i] = mx[i] > m[i] + 8.f ? mx[i] : m[i];  // (from -inf: any score moves it)
        moves |= m_new[i] != m[i];
      }
      if (__any_sync(0xffffffffu, moves)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float a = m_new[i] == m[i] ? 1.f : ex2_approx(m[i] - m_new[i]);
          m[i] = m_new[i];
          l[i] *= a;
#pragma unroll
          for (int n = 0; n < DH / 8; ++n) {
            o[n][2 * i] *= a;
            o[n][2 * i + 1] *= a;
          }
        }
      }
      const float ref[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        uint32_t a[4];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float p0 = ex2_approx(s[g][n][2 * i] - ref[i]), p1 = ex2_approx(s[g][n][2 * i + 1] - ref[i]);
            l[i] += p0 + p1;
            a[2 * n + i] = bf16_pair(p0, p1);
          }
#pragma unroll
        for (int n = 0; n < DH / 8; n += 2) {
          uint32_t f[4];
          ldmatrix_x4_trans(v_tile + C::at((g0 + g) * 16 + ((lane / 8) % 2) * 8 + lane % 8, n + lane / 16), f);
          mma_bf16(o[n], a, f[0], f[1]);
          mma_bf16(o[n + 1], a, f[2], f[3]);
        }
      }
    }
    // ---- end of the piece
    const bool whole = walk.whole();
    const int32_t part = walk.part();
    const int64_t kv_head_bytes = (int64_t)(walk.head / p.per_kv) * p.head_bytes;
    const int32_t k_begin = blk0 * kMmaKeys, k_end = (blk0 + blocks) * kMmaKeys;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
    }
    if constexpr (MW == 1) {
      if (lane % 4 == 0) {
        merge_sums[warp * 16 + row_lo] = make_float2(m[0], l[0]);
        merge_sums[warp * 16 + row_lo + 8] = make_float2(m[1], l[1]);
      }
      __syncthreads();
      float w[2], ref[2], sum[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        ref[i] = -INFINITY;
        for (int x = 0; x < 4; ++x) ref[i] = fmaxf(ref[i], merge_sums[x * 16 + row_lo + 8 * i].x);
        const float r = ref[i] == -INFINITY ? 0.f : ref[i];
        sum[i] = 0.f;
        for (int x = 0; x < 4; ++x) {
          const float2 y = merge_sums[x * 16 + row_lo + 8 * i];
          sum[i] = fmaf(ex2_approx(y.x - r), y.y, sum[i]);
        }
        w[i] = ex2_approx(m[i] - r);
      }
      // one warp after another adds its share; the places are by thread, so each reads and writes its own
      for (int x = 0; x < 4; ++x) {
        if (warp == x) {
#pragma unroll
          for (int n = 0; n < DH / 8; ++n)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              float* to = merge + (n * 4 + c) * 32 + lane;
              const float mine = w[c / 2] * o[n][c];
              *to = x == 0 ? mine : *to + mine;
            }
        }
        __syncthreads();
      }
      if (warp == 0 && lane % 4 == 0) {  // (read above by all, before the barriers)
        merge_sums[row_lo] = make_float2(ref[0], sum[0]);
        merge_sums[row_lo + 8] = make_float2(ref[1], sum[1]);
      }
      __syncthreads();
      for (int32_t row = warp; row < min(rows, 16); row += 4) {
        float acc[DH / 32];
        const float2 ms = merge_sums[row];
        float mm = ms.x, ll = ms.y, probe = ms.y * 0.f;
#pragma unroll
        for (int c = 0; c < DH / 32; ++c) {
          const int col = lane + 32 * c;
          acc[c] = merge[((col / 8) * 4 + (row / 8) * 2 + col % 2) * 32 + (row % 8) * 4 + (col % 8) / 2];
          probe = fmaf(acc[c], 0.f, probe);
        }
        const RowKeys rk = attn_row(p, e, row / p.group);
        const int32_t h = walk.head * p.group + row % p.group;
        if (__any_sync(0xffffffffu, probe != 0.f))
          attn_row_by_hand<DH>(p, e, kv_head_bytes, p.Q + (int64_t)(e.row0 + row / p.group) * p.q_row_bytes + h * p.q_head_bytes, rk,
                               slope_of(p, h), k_begin, k_end, mm, ll, acc);
        if (whole) {
          const float inv = 1.f / ll;
          __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.O + (int64_t)(e.row0 + row / p.group) * p.o_row_bytes + h * p.o_head_bytes);
#pragma unroll
          for (int c = 0; c < DH / 32; ++c) out[lane + 32 * c] = __float2bfloat16_rn(rk.lo < rk.hi ? acc[c] * inv : 0.f);
        } else {
          float* out = attn_part(p, part) + row * DH;
#pragma unroll
          for (int c = 0; c < DH / 32; ++c) out[lane + 32 * c] = acc[c];
          if (lane == 0) attn_part_sums(p, gridDim.x, part)[row] = make_float2(mm, ll);
        }
      }
      __syncthreads();  // the next piece writes there
    } else {
      float probe[2] = {l[0] * 0.f, l[1] * 0.f};
#pragma unroll
      for (int n = 0; n < DH / 8; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) probe[c / 2] = fmaf(o[n][c], 0.f, probe[c / 2]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int32_t row = row_lo + 8 * i;
        const uint32_t quad = 0xfu << (lane & ~3);
        uint32_t bad = __ballot_sync(0xffffffffu, probe[i] != 0.f && row < rows);
        const bool mine = (bad & quad) != 0;
        if (row < rows && !mine) {
          const int32_t h = walk.head * p.group + row % p.group;
          if (whole) {
            const float inv = keys[i].lo < keys[i].hi ? 1.f / l[i] : 0.f;
            uint8_t* out = p.O + (int64_t)(e.row0 + row / p.group) * p.o_row_bytes + h * p.o_head_bytes;
#pragma unroll
            for (int n = 0; n < DH / 8; ++n)
              *reinterpret_cast<uint32_t*>(out + (n * 8 + 2 * (lane % 4)) * 2) = bf16_pair(o[n][2 * i] * inv, o[n][2 * i + 1] * inv);
          } else {
            float* out = attn_part(p, part) + (int64_t)row * DH;
#pragma unroll
            for (int n = 0; n < DH / 8; ++n)
              *reinterpret_cast<float2*>(out + n * 8 + 2 * (lane % 4)) = make_float2(o[n][2 * i], o[n][2 * i + 1]);
            if (lane % 4 == 0) attn_part_sums(p, gridDim.x, part)[row] = make_float2(m[i], l[i]);
          }
        }
        while (bad != 0) {  // a row at a time, by the warp
          const int src = __ffs(bad) - 1;
          bad &= ~(0xfu << (src & ~3));
          const int32_t r = warp * 16 + src / 4 + 8 * i, h = walk.head * p.group + r % p.group;
          const RowKeys rk = attn_row(p, e, r / p.group);
          float acc[DH / 32], mm, ll;
          attn_row_by_hand<DH>(p, e, kv_head_bytes, p.Q + (int64_t)(e.row0 + r / p.group) * p.q_row_bytes + h * p.q_head_bytes, rk,
                               slope_of(p, h), k_begin, k_end, mm, ll, acc);
          if (whole) {
            __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.O + (int64_t)(e.row0 + r / p.group) * p.o_row_bytes + h * p.o_head_bytes);
#pragma unroll
            for (int c = 0; c < DH / 32; ++c) out[lane + 32 * c] = __float2bfloat16_rn(rk.lo < rk.hi ? acc[c] / ll : 0.f);
          } else {
            float* out = attn_part(p, part) + (int64_t)r * DH;
#pragma unroll
            for (int c = 0; c < DH / 32; ++c) out[lane + 32 * c] = acc[c];
            if (lane == 0) attn_part_sums(p, gridDim.x, part)[r] = make_float2(mm, ll);
          }
        }
      }
    }
  }
  cp_async_wait<0>();
}

template <int DH, int MW>
rocs_status_t launch_mma(const CacheAttn& p, int32_t grid, cudaStream_t stream) {
  auto kernel = mma_kernel<DH, MW>;
  ROCS_ALLOW_SMEM(kernel, MmaCfg<DH>::kSmem);
  return launch_dependent(kernel, dim3((unsigned)grid), kMmaThreads, (size_t)MmaCfg<DH>::kSmem, stream, p);
}

}  // namespace

int attn_mma_ctas_per_sm(int32_t dh) {
  return dh == 128 ? MmaCfg<128>::kPerSm : dh == 64 ? MmaCfg<64>::kPerSm : MmaCfg<32>::kPerSm;
}

rocs_status_t attn_mma(const CacheAttn& p, int32_t grid, cudaStream_t stream) {
  const bool few = p.tile_rows == 16;
  if (p.dh == 128) return few ? launch_mma<128, 1>(p, grid, stream) : launch_mma<128, 4>(p, grid, stream);
  if (p.dh == 64) return few ? launch_mma<64, 1>(p, grid, stream) : launch_mma<64, 4>(p, grid, stream);
  return few ? launch_mma<32, 1>(p, grid, stream) : launch_mma<32, 4>(p, grid, stream);
}

}  // namespace rocs
