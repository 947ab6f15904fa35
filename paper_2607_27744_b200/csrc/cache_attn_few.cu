// Attention over the paged cache for tiles of up to 16 rows (bf16): a single event, or a few, of the query heads that share a
// key head.  The time is the reading of K and V, 4 dh flops per row and key of 4 dh bytes.
//
// Five warps.  Warp 4 loads: blocks of 64 keys, page by page through a tensor map whose last dimension is the page, into a
// ring of 3 or 4 stages; it runs ahead over the end of a tile into the next, so the memory is busy while the others finish
// a tile.  Warps 0-3 compute, 16 keys of each block each, on mma.sync m16n8k16 with the KEYS as the 16 rows and the queries
// as the 8 columns: S^T = K Q^T and O^T += V^T P^T.  A single event of 8 query heads then fills the instruction, where the
// other way round half of its rows would be empty, and half the registers hold O.  (P^T needs the transposed fragment of
// S^T: one movmatrix per 8 keys.)  The two to four CTAs of an SM are at different places, which hides what a block's chain of
// loads, products, exponentials and products takes.
//
// Every warp keeps a reference and sums of its own per row; the reference moves when a score passes it by 2^8, which one vote
// per block asks for.  At the end of a piece the four add up through shared memory.
// Probabilities are rounded to bf16 as the second product's operand (half a step, 2^-9 to 2^-8 of each; the plain form does not:
// errors of 2.3e-3 and 1.7e-3 of the values against 64 bits, the result's own rounding among them); their sum is of unrounded ones.
#include <algorithm>

#include "cache_attn.cuh"

namespace rocs {
namespace {

using namespace ptx;

constexpr int kFewThreads = 160;
constexpr uint32_t kStatusFew = 0x600;

template <int DH, int NT>
struct FewCfg {
  static constexpr int kBoxCols = DH < 64 ? DH : 64, kRowBytes = kBoxCols * 2, kBoxes = DH / kBoxCols;
  static constexpr int kBoxBytes = kFewKeys * kRowBytes;
  static constexpr int kTileBytes = kBoxes * kBoxBytes;      // K or V of a block
  static constexpr int kStages = DH == 32 ? 4 : 3;
  static constexpr int kRegs = DH < 64 ? 8 : 16;             // output registers (of 8 rows) that warps exchange at a time
  static constexpr int kRounds = DH / 4 / kRegs;
  static constexpr uint32_t kOffMerge = kStages * 2 * kTileBytes;          // [4 warps][kRegs][32 lanes] fp32
  static constexpr uint32_t kOffSums = kOffMerge + 4 * kRegs * 32 * 4;     // [4 warps][16 rows] reference and sum
  static constexpr uint32_t kFull = kOffSums + 4 * 16 * 8, kEmpty = kFull + 8 * kStages, kMeet = kEmpty + 8 * kStages;
  static constexpr uint32_t kOffAbort = kMeet + 8;
  static constexpr int kSmem = kOffAbort + 8;
  static constexpr int kPerSm = DH == 128 ? 2 : DH == 64 ? 3 : 4;
  static_assert(kPerSm * (kSmem + (int)sizeof(AttnLine) + 2048) <= 228 * 1024, "shared memory of an SM");
  // place of 16-byte vector `chunk` of a key's row under the tensor map's swizzle
  __device__ static uint32_t at(uint32_t key, uint32_t chunk) {
    if constexpr (kRowBytes == 64) return key * 64 + ((chunk ^ ((key >> 1) & 3)) << 4);
    return (chunk >> 3) * kBoxBytes + key * 128 + (((chunk & 7) ^ (key & 7)) << 4);
  }
  // the same for chunk 2 k + c, given at(key, c): an exclusive or inside a box, and tiles begin at multiples of 1024
  __device__ static uint32_t step(uint32_t at_c, int k) {
    constexpr int kPerBox = kBoxCols / 16;
    return (at_c ^ ((k % kPerBox) * 32)) + (k / kPerBox) * kBoxBytes;
  }
};

// What stands for "no reference yet": finite, so that it needs no case of its own.  Scores below it weigh 0; a row that has no
// others is computed again.
constexpr float kNoReference = -3.0e38f;

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
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int32_t x, int32_t y, int32_t z,
                                            int32_t w) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}

// NT: groups of 8 rows (1 or 2); MODS: scores are capped or fall with distance.
template <int DH, int NT, bool MODS>
__global__ void __launch_bounds__(kFewThreads, FewCfg<DH, NT>::kPerSm)
few_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CacheAttn p) {
  using C = FewCfg<DH, NT>;
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ AttnLine line_mem;
  const uint32_t sb = smem_u32(smem);
  AbortFlag* abort_flag = reinterpret_cast<AbortFlag*>(smem + C::kOffAbort);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if ((sb & 1023u) != 0) {  // the swizzled tiles assume a 1024-byte aligned base
    if (threadIdx.x == 0) atomicCAS(p.status, 0u, kStatusFew | 15);
    return;
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(reinterpret_cast<uint64_t*>(smem + C::kFull + 8 * s), 1);
      mbar_init(reinterpret_cast<uint64_t*>(smem + C::kEmpty + 8 * s), 4);
    }
    mbar_init(reinterpret_cast<uint64_t*>(smem + C::kMeet), 4);
    abort_flag->v = 0;
    fence_mbar_init();
    prefetch_tensormap(&map_k);
    prefetch_tensormap(&map_v);
  }
  griddep_wait();
  griddep_launch_dependents();
  const AttnLineView view = attn_line<kFewThreads>(p, line_mem);
  __syncthreads();
  AttnWalk walk;
  if (!walk.start<127>(p, view)) return;
  if (warp == 4) {
    // ------------------------------ loads ------------------------------------------------------
    const int32_t box_rows = min(p.page, kFewKeys), boxes = kFewKeys / box_rows;  // pages (or parts of one) of a block
    uint32_t it = 0;
    bool ok = true;
    for (; ok && walk.more(); walk.next(p, view)) {
      const AttnEntry e = view.entry[walk.entry];
      if (e.blocks == 0) continue;
      const int32_t blk0 = e.blk0 + walk.block0(p), n = walk.blocks(p), kv_head = walk.head / p.per_kv;
      const int32_t* row = p.table + (int64_t)e.slot * p.width;
      auto look_up = [&](int32_t b) {  // page of this lane's box of block b; none behind the slot's end: zeros
        const int32_t j = (blk0 + b) * kFewKeys + lane * box_rows;
        return lane < boxes && j < e.L ? row[page_of(p, j)] : -1;
      };
      int32_t id_next = look_up(0);
      for (int32_t b = 0; b < n; ++b) {
        const int32_t id = id_next;
        if (b + 1 < n) id_next = look_up(b + 1);
        const uint32_t st = it % C::kStages;
        const bool free = mbar_wait_paced(sb + C::kEmpty + 8 * st, ((it / C::kStages) & 1) ^ 1, abort_flag, p.status, kStatusFew | 1);
        if (!__all_sync(0xffffffffu, free)) { ok = false; break; }
        const int32_t j0 = (blk0 + b) * kFewKeys;
        const int32_t in_page = p.page > kFewKeys ? j0 - page_of(p, j0) * p.page : 0;
        const uint32_t bar = sb + C::kFull + 8 * st, dst = sb + st * 2 * C::kTileBytes;
        if (lane == 0) mbar_expect_tx(bar, 2 * C::kTileBytes);
        __syncwarp();
        for (int32_t x = 0; x < boxes; ++x) {
          const int32_t page = __shfl_sync(0xffffffffu, id, x);
          if (elect_one()) {
#pragma unroll
            for (int bx = 0; bx < C::kBoxes; ++bx) {
              const uint32_t to = dst + bx * C::kBoxBytes + x * box_rows * C::kRowBytes;
              tma_load_4d(to, &map_k, bar, bx * C::kBoxCols, in_page, kv_head, page);
              tma_load_4d(to + C::kTileBytes, &map_v, bar, bx * C::kBoxCols, in_page, kv_head, page);
            }
          }
          __syncwarp();
        }
        ++it;
      }
    }
    if (!ok)  // let the loads in flight land before the CTA's shared memory goes away
      for (uint32_t s = 0; s < C::kStages; ++s) {
        const uint32_t issued = it / C::kStages + ((it % C::kStages > s) ? 1 : 0);
        if (issued == 0) continue;
        const uint64_t t0 = globaltimer_ns();
        while (!mbar_try_wait_brief(sb + C::kFull + 8 * s, (issued - 1) & 1) && globaltimer_ns() - t0 < kWaitLimitNs) {}
      }
    return;
  }
  // ------------------------------ compute ------------------------------------------------------
  float* merge = reinterpret_cast<float*>(smem + C::kOffMerge);
  float2* sums = reinterpret_cast<float2*>(smem + C::kOffSums);  // [4 warps][16 rows]
  uint32_t it = 0, n_meet = 0;
  auto meet = [&]() {  // the four warps
    __syncwarp();
    if (lane == 0) mbar_arrive(sb + C::kMeet);
    const bool ok = mbar_wait_paced(sb + C::kMeet, n_meet & 1, abort_flag, p.status, kStatusFew | 2);
    ++n_meet;
    return __all_sync(0xffffffffu, ok) != 0;
  };
  const uint32_t k_place = C::at(warp * 16 + lane % 8 + ((lane / 8) & 1) * 8, lane / 16);
  const uint32_t v_place = C::at(warp * 16 + lane % 8 + (lane / 16) * 8, (lane / 8) & 1);
  // what a piece needs from memory, fetched while the piece in front is computed
  uint32_t q_next[NT][DH / 16][2];
  auto fetch = [&](const AttnWalk& w) {
    if (!w.more()) return;
    const AttnEntry& e = view.entry[w.entry];
    const int32_t rows = e.count * p.group;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int32_t row = n * 8 + lane / 4;
      const bool there = row < rows;
      const uint8_t* src = p.Q;
      if (there) src += (int64_t)(e.row0 + row / p.group) * p.q_row_bytes + (w.head * p.group + row % p.group) * p.q_head_bytes;
#pragma unroll
      for (int k = 0; k < DH / 16; ++k)
#pragma unroll
        for (int c = 0; c < 2; ++c)
          q_next[n][k][c] = there ? *reinterpret_cast<const uint32_t*>(src + (k * 16 + c * 8 + 2 * (lane % 4)) * 2) : 0u;
    }
  };
  fetch(walk);
  AttnWalk after = walk;
  for (; walk.more(); walk.next(p, view)) {
    const AttnEntry e = view.entry[walk.entry];
    const int32_t rows = e.count * p.group;
    uint32_t q[NT][DH / 16][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int k = 0; k < DH / 16; ++k) {
        q[n][k][0] = q_next[n][k][0];
        q[n][k][1] = q_next[n][k][1];
      }
    after.next(p, view);
    fetch(after);
    // this lane's columns: rows n * 8 + 2 (lane % 4) + i
    int32_t lo[NT][2], hi[NT][2];
    int32_t pos[NT][2];
    float slope[NT][2], m[NT][2], l[NT][2];
    int32_t lo_most = 0, hi_least = 0x7fffffff;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int32_t row = n * 8 + 2 * (lane % 4) + i;
        RowKeys rk{0, 0x7fffffff, 0};  // a row that does not exist asks for no mask
        slope[n][i] = 0.f;
        if (row < rows) {
          rk = attn_row(p, e, row / p.group);
          if (MODS) slope[n][i] = slope_of(p, walk.head * p.group + row % p.group);
        }
        lo[n][i] = rk.lo;
        hi[n][i] = rk.hi;
        pos[n][i] = rk.pos;
        lo_most = max(lo_most, rk.lo);
        hi_least = min(hi_least, rk.hi);
        m[n][i] = kNoReference;
        l[n][i] = 0.f;
      }
    lo_most = __reduce_max_sync(0xffffffffu, lo_most);
    hi_least = __reduce_min_sync(0xffffffffu, hi_least);
    float o[NT][DH / 16][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int t = 0; t < DH / 16; ++t)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[n][t][c] = 0.f;
    const int32_t blk0 = e.blk0 + walk.block0(p), blocks = e.blocks > 0 ? walk.blocks(p) : 0;
    for (int32_t b = 0; b < blocks; ++b) {
      const uint32_t st = it % C::kStages;
      const bool there = mbar_wait_paced(sb + C::kFull + 8 * st, (it / C::kStages) & 1, abort_flag, p.status, kStatusFew | 3);
      if (!__all_sync(0xffffffffu, there)) return;
      ++it;
      const uint32_t k_tile = sb + st * 2 * C::kTileBytes, v_tile = k_tile + C::kTileBytes;
      const int32_t key0 = warp * 16, j0 = (blk0 + b) * kFewKeys + key0;  // this warp's keys
      if (j0 >= e.L) {  // nothing there (the slot's last block): nor is anything added
        __syncwarp();
        if (lane == 0) mbar_arrive(sb + C::kEmpty + 8 * st);
        continue;
      }
      float s[NT][2][4];  // two chains of products each
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[n][0][c] = s[n][1][c] = 0.f;
      const uint32_t k_at = k_tile + k_place, v_at = v_tile + v_place;
#pragma unroll
      for (int k = 0; k < DH / 16; ++k) {
        uint32_t a[4];
        ldmatrix_x4(C::step(k_at, k), a);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_bf16(s[n][k & 1], a, q[n][k][0], q[n][k][1]);
      }
      float x[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) x[n][c] = (s[n][0][c] + s[n][1][c]) * p.scale;
      if (MODS) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float away = (float)(pos[n][i] - j0 - lane / 4);
#pragma unroll
            for (int c = i; c < 4; c += 2) {
              if (p.cap > 0.f) x[n][c] = p.cap * tanh_of(x[n][c]);
              x[n][c] = fmaf(-slope[n][i], fabsf(away - (c / 2) * 8), x[n][c]);
            }
          }
      }
      if (!(j0 >= lo_most && j0 + 16 <= hi_least)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int32_t j = j0 + lane / 4 + (c / 2) * 8;
            if (j < lo[n][c % 2] || j >= hi[n][c % 2]) x[n][c] = -INFINITY;
          }
      }
      bool moves = false;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) moves |= x[n][c] > m[n][c % 2] + 8.f;  // (any score passes kNoReference)
      if (__any_sync(0xffffffffu, moves)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float mx = fmaxf(x[n][i], x[n][2 + i]);
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
            const float m_new = mx > m[n][i] + 8.f ? mx : m[n][i];  // a row's own decision
            const float f = m_new == m[n][i] ? 1.f : ex2_approx(m[n][i] - m_new);
            m[n][i] = m_new;
            l[n][i] *= f;
#pragma unroll
            for (int t = 0; t < DH / 16; ++t) {
              o[n][t][i] *= f;
              o[n][t][2 + i] *= f;
            }
          }
      }
      uint32_t pb[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float p0 = ex2_approx(x[n][0] - m[n][0]), p1 = ex2_approx(x[n][1] - m[n][1]), p2 = ex2_approx(x[n][2] - m[n][0]),
                    p3 = ex2_approx(x[n][3] - m[n][1]);
        l[n][0] += p0 + p2;
        l[n][1] += p1 + p3;
        pb[n][0] = transposed(bf16_pair(p0, p1));
        pb[n][1] = transposed(bf16_pair(p2, p3));
      }
      if (j0 + 16 > e.L) {  // what the last page holds behind the slot's end may be anything, and 0 x NaN is not 0
#pragma unroll 1
        for (int32_t x = lane; x < (j0 + 16 - e.L) * (DH / 8); x += 32)
          *reinterpret_cast<uint4*>(smem + (v_tile - sb) + C::at(key0 + (e.L - j0) + x / (DH / 8), x % (DH / 8))) = make_uint4(0u, 0u, 0u, 0u);
        fence_proxy_async_smem();  // (the place is loaded into again)
        __syncwarp();
      }
#pragma unroll
      for (int t = 0; t < DH / 16; ++t) {
        uint32_t a[4];
        ldmatrix_x4_trans(C::step(v_at, t), a);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_bf16(o[n][t], a, pb[n][0], pb[n][1]);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(sb + C::kEmpty + 8 * st);
    }
    // ---- end of the piece: the four warps' sums and outputs
    const bool whole = walk.whole();
    const int32_t part = walk.part();
    const int64_t kv_head_bytes = (int64_t)(walk.head / p.per_kv) * p.head_bytes;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], d);
        if (lane / 4 == 0) sums[warp * 16 + n * 8 + 2 * lane + i] = make_float2(m[n][i], l[n][i]);
      }
    if (!meet()) return;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float f[2], acc[2][DH / 32];  // this warp's rows of the 8: warp and warp + 4
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float ref = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) ref = fmaxf(ref, sums[w * 16 + n * 8 + 2 * (lane % 4) + i].x);
        f[i] = ex2_approx(m[n][i] - ref);
      }
#pragma unroll
      for (int u = 0; u < C::kRounds; ++u) {
        if ((n > 0 || u > 0) && !meet()) return;  // the exchange in front has been read
#pragma unroll
        for (int x = 0; x < C::kRegs; ++x) {
          const int reg = u * C::kRegs + x;
          merge[(warp * C::kRegs + x) * 32 + lane] = f[reg % 2] * o[n][reg / 4][reg % 4];
        }
        if (!meet()) return;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = warp + 4 * i;
#pragma unroll
          for (int c = u * C::kRegs / 8; c < (u + 1) * C::kRegs / 8; ++c) {
            const int d = lane + 32 * c, reg = (d / 16) * 4 + ((d % 16) / 8) * 2 + r % 2 - u * C::kRegs, from = (d % 8) * 4 + r / 2;
            acc[i][c] = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) acc[i][c] += merge[(w * C::kRegs + reg) * 32 + from];
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int32_t row = n * 8 + warp + 4 * i;
        if (row >= rows) continue;
        const int32_t t = row / p.group, h = walk.head * p.group + row % p.group;
        float mm = -INFINITY, ll = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) mm = fmaxf(mm, sums[w * 16 + row].x);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float2 y = sums[w * 16 + row];
          ll = fmaf(ex2_approx(y.x - mm), y.y, ll);
        }
        float probe = ll * 0.f;
#pragma unroll
        for (int c = 0; c < DH / 32; ++c) probe = fmaf(acc[i][c], 0.f, probe);
        const RowKeys rk = attn_row(p, e, t);
        if (__any_sync(0xffffffffu, probe != 0.f || ll == 0.f))
          attn_row_by_hand<DH>(p, e, kv_head_bytes, p.Q + (int64_t)(e.row0 + t) * p.q_row_bytes + h * p.q_head_bytes, rk, slope_of(p, h),
                               blk0 * kFewKeys, (blk0 + blocks) * kFewKeys, mm, ll, acc[i]);
        if (whole) {
          const float inv = 1.f / ll;
          __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.O + (int64_t)(e.row0 + t) * p.o_row_bytes + h * p.o_head_bytes);
#pragma unroll
          for (int c = 0; c < DH / 32; ++c) out[lane + 32 * c] = __float2bfloat16_rn(rk.lo < rk.hi ? acc[i][c] * inv : 0.f);
        } else {
          float* out = attn_part(p, part) + row * DH;
#pragma unroll
          for (int c = 0; c < DH / 32; ++c) out[lane + 32 * c] = acc[i][c];
          if (lane == 0) attn_part_sums(p, gridDim.x, part)[row] = make_float2(mm, ll);
        }
      }
    }
    if (!meet()) return;  // the next piece writes there
  }
}

template <int DH, int NT, bool MODS>
rocs_status_t launch_few(const CacheAttn& p, const CUtensorMap& k, const CUtensorMap& v, int32_t grid, cudaStream_t stream) {
  auto kernel = few_kernel<DH, NT, MODS>;
  ROCS_ALLOW_SMEM(kernel, (FewCfg<DH, NT>::kSmem));
  return launch_dependent(kernel, dim3((unsigned)grid), kFewThreads, (size_t)FewCfg<DH, NT>::kSmem, stream, k, v, p);
}
template <int DH>
rocs_status_t few_of(const CacheAttn& p, const CUtensorMap& k, const CUtensorMap& v, int32_t grid, cudaStream_t stream) {
  const bool mods = p.cap > 0.f || p.slopes != nullptr;
  if (p.rows_per_tile * p.group <= 8) return mods ? launch_few<DH, 1, true>(p, k, v, grid, stream) : launch_few<DH, 1, false>(p, k, v, grid, stream);
  return mods ? launch_few<DH, 2, true>(p, k, v, grid, stream) : launch_few<DH, 2, false>(p, k, v, grid, stream);
}

}  // namespace

bool attn_few_supported(int32_t dh, int32_t page) {
  return (dh == 32 || dh == 64 || dh == 128) && (page % kFewKeys == 0 || page == 32 || page == 16 || page == 8);
}
int attn_few_ctas_per_sm(int32_t dh) { return dh == 128 ? FewCfg<128, 2>::kPerSm : dh == 64 ? FewCfg<64, 2>::kPerSm : FewCfg<32, 2>::kPerSm; }

rocs_status_t attn_few(const CacheAttn& p, int32_t H_kv, int32_t grid, cudaStream_t stream) {
  CUtensorMap k, v;
  if (!make_page_map(&k, p.K, p, H_kv, kFewKeys) || !make_page_map(&v, p.V, p, H_kv, kFewKeys)) return ROCS_ERR_CUDA;
  return p.dh == 128 ? few_of<128>(p, k, v, grid, stream) : p.dh == 64 ? few_of<64>(p, k, v, grid, stream) : few_of<32>(p, k, v, grid, stream);
}

}  // namespace rocs
