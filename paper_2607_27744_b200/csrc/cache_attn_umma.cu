// Attention over the paged cache on tcgen05 (bf16, heads of 64 or 128): tiles of 256 rows, two sides of 128 that share the
// key and value blocks of 128 keys in shared memory.  A tile of up to 128 rows has both sides on the same rows, each with
// every other block of keys.
//
// 20 warps:  0-7 and 8-15  softmax of sides A and B, two threads per row: each has 64 of a block's 128 columns
//            16            loads Q and the K blocks, page by page through a tensor map whose last dimension is the page
//            17            loads the V blocks, and zeroes what the last page holds behind the slot's end
//            18            issues the products: S = Q K^T (operands in shared memory) and O += P V (P in tensor memory)
//
// Tensor memory: S of both sides (128 columns each), O of both sides.  P (bf16 pairs) takes the place of the S that it comes
// from, each half of a row in its own half of the columns; the products of a side are issued in the order P_j V_j, S_{j+1},
// and run in that order, so nobody waits for the columns to come free, and the arrival of S_{j+1} says that O holds
// everything up to P_j V_j.  P_j is announced in two parts: the products of the first begin while the second is made.  While
// a side's products run, the other side's softmax does: the products of a block pair take 2048 cycles (heads of 128) and its
// exponentials the same, so what bounds the kernel is how well the two overlap.
//
// Blocks go from the last key to the first: masks (the chunk's own keys) come first, and a score that falls with distance
// is largest there.  A row's reference is the maximum of the first block in which it sees a key; other blocks need no
// maximum.  It moves up where a block's sum passes 2^40, by that sum's exponent, before the next block: both threads of the
// row read what the other's half summed to, and scale O and their sums by the same power of two.  A probability keeps its
// 8 bits wherever the reference is, sums are fp32.  All decisions are a row's own: its bits do not depend on other rows'
// values.
//
// A row whose scores pass its reference by more than fp32's range within one block, or whose masked keys hold NaN or Inf
// values (weight 0, but 0 x Inf is not 0), comes out non-finite and is computed again from the keys that it sees, by a warp.
// So is one whose weights sum to next to nothing (scores of 2^30 and more, see there).
#include <algorithm>
#include <type_traits>

#include "cache_attn.cuh"

namespace rocs {
namespace {

using namespace ptx;

constexpr int kSoftmaxWarps = 16, kLoadK = 16, kLoadV = 17, kIssue = 18;
constexpr int kUmmaThreads = 20 * 32;
constexpr int kSide = 128;               // rows of a side = tensor memory lanes
constexpr int BK = kUmmaKeys;
constexpr uint32_t kStatusCache = 0x500;
constexpr float kMoveAt = 1099511627776.f;  // 2^40

template <int DH_>
struct UmmaCfg {
  static constexpr int DH = DH_;
  static constexpr int kBoxes = DH / 64;                    // operand tiles are boxes of 64 columns, 128-byte rows
  static constexpr int kBoxBytes = 128 * 128;               // 128 rows (queries or keys) of a box
  static constexpr int kTileBytes = kBoxes * kBoxBytes;     // a side's Q, a K block, a V block
  static constexpr int kStages = DH == 128 ? 2 : 4;         // of K and of V
  static constexpr uint32_t kOffQ = 0;
  static constexpr uint32_t kOffK = kOffQ + 2 * kTileBytes;
  static constexpr uint32_t kOffV = kOffK + kStages * kTileBytes;
  static constexpr uint32_t kOffSum = kOffV + kStages * kTileBytes;   // [4 blocks][2 sides][2 halves][128] sums of a block
  static constexpr uint32_t kOffMax = kOffSum + 16 * kSide * 4;       // [2 sides][2 halves][128] maxima of a block
  static constexpr uint32_t kOffEnd = kOffMax + 4 * kSide * 4;        // [2 sides][2 halves][128] (reference, sum, probe, -)
  static constexpr uint32_t kOffBar = kOffEnd + 4 * kSide * 16;
  static constexpr uint32_t kQFull = kOffBar, kQEmpty = kQFull + 8, kSFull = kQEmpty + 8, kPFull = kSFull + 16,
                            kPHalf = kPFull + 16, kOFull = kPHalf + 16, kTail = kOFull + 16, kDrain = kTail + 8, kPair = kDrain + 8, kQuad = kPair + 64, kKFull = kQuad + 32,
                            kKEmpty = kKFull + 8 * kStages,
                            kVFull = kKEmpty + 8 * kStages, kVEmpty = kVFull + 8 * kStages, kOffTmem = kVEmpty + 8 * kStages,
                            kOffAbort = kOffTmem + 8;
  static constexpr int kSmem = kOffAbort + 8;
  static constexpr uint32_t kColO = 256;                    // O of side s at 256 + s * DH
  static_assert(kSmem + (int)sizeof(AttnLine) + 1024 <= 227 * 1024, "shared memory of one SM");
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int32_t x, int32_t y, int32_t z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z)
      : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int32_t x, int32_t y, int32_t z,
                                            int32_t w) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]: A holds bf16 pairs in 32-bit columns (16 keys = 8 columns).
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// A wait that leaves the issue slots to the other warps: a probe may be suspended until the phase completes (0.2 ms at most,
// so that the abort flag is seen).  The softmax waits a good part of a block, and probes that come back at once, with a look
// at the clock between two, cost the long chunk 8 % on a GPU that has not come to its power limit.
__device__ __forceinline__ bool mbar_wait_suspended(uint32_t bar, uint32_t parity, AbortFlag* abort_flag, uint32_t* status, uint32_t code) {
  const uint64_t t0 = globaltimer_ns();
  while (true) {
    uint32_t ok;
    asm volatile(
        "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(ok)
        : "r"(bar), "r"(parity), "r"(200000u)
        : "memory");
    if (ok) return true;
    if (abort_flag->v) return false;
    if (globaltimer_ns() - t0 > kWaitLimitNs) {
      abort_flag->v = 1;
      atomicCAS(status, 0u, code);
      return false;
    }
  }
}
__device__ __forceinline__ void tmem_st_x8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ uint64_t fadd2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

__device__ __forceinline__ uint64_t fmul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// tanh of a pair within [-3/4, 3/4] as t P(t^2) (two instructions of the special-function unit per value and a third for its
// weight would be three times what the kernel waits for without a cap).  `u` receives t^2.  SHORT: fitted for the least absolute
// error, 3.6e-6, which a score has cap times: for caps of up to kShortCap, where that is 2.3e-4, an eighth of what rounding its
// weight to bf16 changes it by.  Otherwise tanh_of's, right to 1.3e-7 of its value whatever the cap (first visits, cap 30: 133 us
// with the short one, 142 us with the long one; candidates, cap 30: 162 and 178 us).
template <bool SHORT>
__device__ __forceinline__ uint64_t tanh_pair(uint64_t t, uint64_t& u) {
  u = fmul2(t, t);
  if constexpr (SHORT) {
    uint64_t r = ffma2(u, pack2(-0.03377828374505043f, -0.03377828374505043f), pack2(0.1257709264755249f, 0.1257709264755249f));
    r = ffma2(r, u, pack2(-0.3322276473045349f, -0.3322276473045349f));
    r = ffma2(r, u, pack2(0.9999555945396423f, 0.9999555945396423f));
    return fmul2(r, t);
  }
  uint64_t r = ffma2(u, pack2(kTanh5, kTanh5), pack2(kTanh4, kTanh4));
  r = ffma2(r, u, pack2(kTanh3, kTanh3));
  r = ffma2(r, u, pack2(kTanh2, kTanh2));
  r = ffma2(r, u, pack2(kTanh1, kTanh1));
  return fmul2(ffma2(r, u, pack2(1.f, 1.f)), t);
}
constexpr float kTanhRange2 = kTanhRange * kTanhRange;
__device__ __forceinline__ float fmax3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// Four lanes with four 16-byte pieces of a row each: lane c of them gets piece c of all four rows, so that a store of the warp
// touches 8 rows with 64 bytes each and not 32 with 16.
__device__ __forceinline__ void swap_pieces(uint4& mine, uint4& other, bool upper, int distance) {
  const uint4 give = upper ? mine : other;
  uint4 got;
  got.x = __shfl_xor_sync(0xffffffffu, give.x, distance);
  got.y = __shfl_xor_sync(0xffffffffu, give.y, distance);
  got.z = __shfl_xor_sync(0xffffffffu, give.z, distance);
  got.w = __shfl_xor_sync(0xffffffffu, give.w, distance);
  if (upper) mine = got; else other = got;
}
__device__ __forceinline__ void transpose_pieces(uint4 (&v)[4], int lane) {
  swap_pieces(v[0], v[1], lane & 1, 1);
  swap_pieces(v[2], v[3], lane & 1, 1);
  swap_pieces(v[0], v[2], lane & 2, 2);
  swap_pieces(v[1], v[3], lane & 2, 2);
}

// 2^-n for n >= 0, with the denormal numbers below 2^-126.
__device__ __forceinline__ float exp2_down(int32_t n) {
  return __uint_as_float(n < 127 ? (uint32_t)(127 - n) << 23 : n < 150 ? 1u << (149 - n) : 0u);
}

// 2^x for a pair on the FMA pipes: 2^n 2^f with n the nearest integer and a polynomial of degree 3 for 2^f on [-1/2, 1/2]
// (fitted for the least relative error, 7.5e-5: a 26th of the rounding to bf16 that follows).  Below 2^-125 it stays there;
// what is NaN, or too large for fp32, comes out as NaN, or so large that bf16 has an infinity for it.
__device__ __forceinline__ uint64_t exp2_pair(uint64_t x2) {
  float x0, x1;
  unpack2(x2, x0, x1);
  // (fminf first: it takes NaN to 129, and 2^129 by the addition to the exponent is NaN)
  const uint64_t x = pack2(fmaxf(fminf(x0, 129.f), -125.f), fmaxf(fminf(x1, 129.f), -125.f));
  constexpr float kMagic = 12582912.f;  // 1.5 x 2^23: the sum's last bits are the nearest integer
  const uint64_t t = fadd2(x, pack2(kMagic, kMagic));
  const uint64_t f = fadd2(x, ffma2(t, pack2(-1.f, -1.f), pack2(kMagic, kMagic)));
  uint64_t r = ffma2(f, pack2(0.0551716685295105f, 0.0551716685295105f), pack2(0.2426111251115799f, 0.2426111251115799f));
  r = ffma2(r, f, pack2(0.6932609677314758f, 0.6932609677314758f));
  r = ffma2(r, f, pack2(0.9999280571937561f, 0.9999280571937561f));
  float t0, t1, r0, r1;
  unpack2(t, t0, t1);
  unpack2(r, r0, r1);
  return pack2(__uint_as_float(__float_as_uint(r0) + (__float_as_uint(t0) << 23)),
               __uint_as_float(__float_as_uint(r1) + (__float_as_uint(t1) << 23)));
}

// CAP: 0 none, 1 up to kShortCap, 2 any.
template <int DH, int CAP, bool BIAS>
__global__ void __launch_bounds__(kUmmaThreads, 1)
umma_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
            const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CacheAttn p) {
  using C = UmmaCfg<DH>;
  constexpr int kStages = C::kStages;
  // How many of a half's four groups of 16 keys are announced when their P is there, in front of the others (0: all at once): their
  // products run while the others' exponentials do.  Long chunk: none 500 us, one 499, two 481, three 482; candidates 127.0 and
  // 126.2 with two; capped scores wait longer for a second arrival than they gain (first visits 131.8 and 133.9).
  constexpr int kFirst = CAP ? 0 : 2;
  extern __shared__ __align__(1024) uint8_t smem[];
  __shared__ AttnLine line_mem;
  const uint32_t sb = smem_u32(smem);
  AbortFlag* abort_flag = reinterpret_cast<AbortFlag*>(smem + C::kOffAbort);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if ((sb & 1023u) != 0) {  // the swizzled tiles assume a 1024-byte aligned base
    if (threadIdx.x == 0) atomicCAS(p.status, 0u, kStatusCache | 15);
    return;
  }
  if (threadIdx.x == 0) {
    auto init = [&](uint32_t off, int n, uint32_t count) {
      for (int x = 0; x < n; ++x) mbar_init(reinterpret_cast<uint64_t*>(smem + off + 8 * x), count);
    };
    init(C::kQFull, 1, 1);
    init(C::kQEmpty, 1, 1);
    init(C::kSFull, 2, 1);
    init(C::kPFull, 2, 8);
    init(C::kPHalf, 2, 8);
    init(C::kOFull, 2, 1);
    init(C::kTail, 1, 1);
    init(C::kDrain, 1, 1);
    init(C::kPair, 8, 2);
    init(C::kQuad, 4, 4);
    init(C::kKFull, kStages, 1);
    init(C::kKEmpty, kStages, 1);
    init(C::kVFull, kStages, 1);
    init(C::kVEmpty, kStages, 1);
    abort_flag->v = 0;
    fence_mbar_init();
  }
  if (warp == kIssue) {
    tmem_alloc(reinterpret_cast<uint32_t*>(smem + C::kOffTmem), 512);
    tmem_relinquish();
  }
  if (warp == kLoadK && lane == 0) {
    prefetch_tensormap(&map_q);
    prefetch_tensormap(&map_k);
    prefetch_tensormap(&map_v);
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *reinterpret_cast<const uint32_t*>(smem + C::kOffTmem);
  griddep_wait();
  griddep_launch_dependents();
  const AttnLineView view = attn_line<kUmmaThreads>(p, line_mem);
  AttnWalk walk;
  const bool any = walk.start<kUmmaThreads - 1>(p, view);
  const int32_t per_side = p.rows_per_tile / 2;  // batch rows of a side

  if (!any) {
    // no work: straight to the end
  } else if (warp == kLoadK || warp == kLoadV) {
    // ------------------------------ loads ------------------------------------------------------
    const bool is_k = warp == kLoadK;
    const CUtensorMap* map = is_k ? &map_k : &map_v;
    const uint32_t full = sb + (is_k ? C::kKFull : C::kVFull), empty = sb + (is_k ? C::kKEmpty : C::kVEmpty);
    const uint32_t dst0 = sb + (is_k ? C::kOffK : C::kOffV);
    const int32_t box_rows = min(p.page, BK), boxes = BK / box_rows;  // pages (or parts of one) of a block
    uint32_t it = 0, n_piece = 0, n_tail = 0;
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity, uint32_t code) {
      return __all_sync(0xffffffffu, mbar_wait_paced(bar, parity, abort_flag, p.status, kStatusCache | code)) != 0;
    };
    for (; ok && walk.more(); walk.next(p, view)) {
      const AttnEntry e = view.entry[walk.entry];
      if (e.blocks == 0) continue;
      const int32_t blk0 = e.blk0 + walk.block0(p), n = walk.blocks(p), kv_head = walk.head / p.per_kv;
      const int32_t* row = p.table + (int64_t)e.slot * p.width;
      auto look_up = [&](int32_t b) {  // page of this lane's box of block b; none behind the slot's end: zeros
        const int32_t j = (blk0 + b) * BK + lane * box_rows;
        return lane < boxes && j < e.L ? row[page_of(p, j)] : -1;
      };
      int32_t id_next = look_up(n - 1);
      if (is_k) {
        if (!wait(sb + C::kQEmpty, (n_piece & 1) ^ 1, 1)) { ok = false; break; }
        const int sides = e.count > per_side ? 2 : 1;
        if (elect_one()) {
          const uint32_t bytes = (uint32_t)(per_side * p.group) * 128u * C::kBoxes;
          mbar_expect_tx(sb + C::kQFull, sides * bytes);
          for (int s = 0; s < sides; ++s)
#pragma unroll
            for (int bx = 0; bx < C::kBoxes; ++bx)
              tma_load_3d(sb + C::kOffQ + s * C::kTileBytes + bx * C::kBoxBytes, &map_q, sb + C::kQFull, bx * 64, walk.head * p.group,
                          e.row0 + s * per_side);
        }
        __syncwarp();
      }
      ++n_piece;
      for (int32_t b = n - 1; b >= 0; --b) {
        const int32_t id = id_next;
        if (b > 0) id_next = look_up(b - 1);
        const uint32_t st = it % kStages;
        if (!wait(empty + 8 * st, ((it / kStages) & 1) ^ 1, is_k ? 2 : 3)) { ok = false; break; }
        const int32_t j0 = (blk0 + b) * BK;
        const int32_t in_page = p.page > BK ? j0 - page_of(p, j0) * p.page : 0;
        // what the slot's last page holds behind its end may be anything, and 0 x NaN is not 0: such a V block lands on a
        // barrier of the loader's own, which zeroes the rest of the page and then passes the block on
        const bool tail = !is_k && j0 + BK > e.L && e.L % p.page != 0;
        const uint32_t landed = tail ? sb + C::kTail : full + 8 * st;
        if (lane == 0) mbar_expect_tx(landed, C::kTileBytes);
        __syncwarp();
        for (int32_t x = 0; x < boxes; ++x) {
          const int32_t page = __shfl_sync(0xffffffffu, id, x);
          if (elect_one()) {
#pragma unroll
            for (int bx = 0; bx < C::kBoxes; ++bx)
              tma_load_4d(dst0 + st * C::kTileBytes + bx * C::kBoxBytes + x * box_rows * 128, map, landed, bx * 64, in_page, kv_head,
                          page);
          }
          __syncwarp();
        }
        if (tail) {
          if (!wait(landed, n_tail & 1, 4)) { ok = false; break; }
          ++n_tail;
          const int32_t first = e.L - j0, last = min((e.L + p.page - 1) / p.page * p.page - j0, BK);
          uint8_t* v = smem + C::kOffV + st * C::kTileBytes;
          for (int bx = 0; bx < C::kBoxes; ++bx)
            for (int32_t x = first * 8 + lane; x < last * 8; x += 32)
              *reinterpret_cast<uint4*>(v + bx * C::kBoxBytes + x * 16) = make_uint4(0u, 0u, 0u, 0u);
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(full + 8 * st);
        }
        ++it;
      }
    }
    if (!ok) {  // let the loads in flight land before the CTA's shared memory goes away
      for (uint32_t s = 0; s < kStages; ++s) {
        const uint32_t issued = it / kStages + ((it % kStages > s) ? 1 : 0);
        if (issued == 0) continue;
        const uint64_t t0 = globaltimer_ns();
        while (!mbar_try_wait_brief(full + 8 * s, (issued - 1) & 1) && globaltimer_ns() - t0 < kWaitLimitNs) {}
      }
      if (is_k && n_piece > 0) {
        const uint64_t t0 = globaltimer_ns();
        while (!mbar_try_wait_brief(sb + C::kQFull, (n_piece - 1) & 1) && globaltimer_ns() - t0 < kWaitLimitNs) {}
      }
    }
  } else if (warp == kIssue) {
    // ------------------------------ products: one thread ---------------------------------------
    if (elect_one()) {
      constexpr uint32_t idesc_s = umma_idesc_bf16(kSide, BK, false, false);  // S = Q K^T, both K-major
      constexpr uint32_t idesc_o = umma_idesc_bf16(kSide, DH, false, true);   // O = P V, V is MN-major
      const uint64_t dq = smem_desc_sw128(sb + C::kOffQ, 1024, 16);
      const uint64_t dk = smem_desc_sw128(sb + C::kOffK, 1024, 16);
      const uint64_t dv = smem_desc_sw128(sb + C::kOffV, 1024, C::kBoxes > 1 ? C::kBoxBytes : 16);
      uint32_t kt = 0, vt = 0, n_piece = 0, cnt_p[2] = {0, 0};
      bool ok = true;
      auto wait = [&](uint32_t bar, uint32_t parity, uint32_t code) {
        if (!mbar_wait_paced(bar, parity, abort_flag, p.status, kStatusCache | code)) ok = false;
        return ok;
      };
      auto issue_s = [&](int side, int q_side, uint32_t st) {
#pragma unroll
        for (int k = 0; k < DH / 16; ++k)
          umma_ss(tmem + side * 128, dq + q_side * (C::kTileBytes >> 4) + (k / 4) * (C::kBoxBytes >> 4) + 2 * (k % 4),
                  dk + st * (C::kTileBytes >> 4) + (k / 4) * (C::kBoxBytes >> 4) + 2 * (k % 4), idesc_s, k != 0 ? 1u : 0u);
        umma_commit(sb + C::kSFull + 8 * side);
      };
      // 16 keys of P: 8 columns, in their half of the row's S; keys [from, to) x 16 of either half
      auto issue_pv = [&](int side, uint32_t st, bool first, auto from, auto to) {
#pragma unroll
        for (int k = 0; k < BK / 16; ++k)
          if (k % 4 >= decltype(from)::value && k % 4 < decltype(to)::value)
            umma_ts(tmem + C::kColO + side * DH, tmem + side * 128 + (k / 4) * 64 + (k % 4) * 8,
                    dv + st * (C::kTileBytes >> 4) + k * (16 * 128 / 16), idesc_o, first && k == 0 ? 0u : 1u);
      };
      auto wait_k = [&]() { return wait(sb + C::kKFull + 8 * (kt % kStages), (kt / kStages) & 1, 6); };
      auto wait_v = [&]() { return wait(sb + C::kVFull + 8 * (vt % kStages), (vt / kStages) & 1, 8); };
      auto wait_p = [&](int side, bool half) {
        if (!wait(sb + (half ? C::kPHalf : C::kPFull) + 8 * side, cnt_p[side] & 1, 7)) return false;
        if (!half) ++cnt_p[side];
        return true;
      };
      auto add_pv = [&](int side, uint32_t st, bool first) {  // false: P did not come
        using std::integral_constant;
        if (kFirst > 0) {
          if (!wait_p(side, true)) return false;
          tc_fence_after_sync();
          issue_pv(side, st, first, integral_constant<int, 0>(), integral_constant<int, kFirst>());
        }
        if (!wait_p(side, false)) return false;
        tc_fence_after_sync();
        issue_pv(side, st, first, integral_constant<int, kFirst>(), integral_constant<int, 4>());
        return true;
      };
      auto k_done = [&]() { umma_commit(sb + C::kKEmpty + 8 * (kt++ % kStages)); };
      auto v_done = [&]() { umma_commit(sb + C::kVEmpty + 8 * (vt++ % kStages)); };
      for (; ok && walk.more(); walk.next(p, view)) {
        const AttnEntry e = view.entry[walk.entry];
        if (e.blocks == 0) continue;
        const int32_t n = walk.blocks(p);
        if (!wait(sb + C::kQFull, n_piece & 1, 5)) break;
        ++n_piece;
        if (e.count > per_side) {  // two sides, every block for both
          if (!wait_k()) break;
          tc_fence_after_sync();
          issue_s(0, 0, kt % kStages);
          issue_s(1, 1, kt % kStages);
          k_done();
          if (n == 1) umma_commit(sb + C::kQEmpty);
          for (int32_t i = 0; i < n && ok; ++i) {
            for (int s = 0; s < 2; ++s) {
              if (s == 0 && (!wait_v() || (i + 1 < n && !wait_k()))) break;  // long there, as a rule: not behind the wait for P
              if (!add_pv(s, vt % kStages, i == 0)) break;
              if (i + 1 < n) issue_s(s, s, kt % kStages);
              else umma_commit(sb + C::kOFull + 8 * s);
            }
            if (!ok) break;
            v_done();
            if (i + 1 < n) {
              k_done();
              if (i + 2 == n) umma_commit(sb + C::kQEmpty);  // the piece's last S
            }
          }
        } else {  // the same rows on both sides, every other block each
          for (int s = 0; s < 2 && s < n; ++s) {
            if (!wait_k()) break;
            tc_fence_after_sync();
            issue_s(s, 0, kt % kStages);
            k_done();
          }
          if (!ok) break;
          if (n <= 2) umma_commit(sb + C::kQEmpty);
          for (int32_t i = 0; i < n; ++i) {
            const int s = i & 1;
            if (!wait_v() || (i + 2 < n && !wait_k()) || !add_pv(s, vt % kStages, i < 2)) break;
            v_done();
            if (i + 2 < n) {
              issue_s(s, 0, kt % kStages);
              k_done();
              if (i + 3 == n) umma_commit(sb + C::kQEmpty);
            } else {
              umma_commit(sb + C::kOFull + 8 * s);
            }
          }
        }
      }
      if (!ok) {
        umma_commit(sb + C::kDrain);
        const uint64_t t0 = globaltimer_ns();
        while (!mbar_try_wait_brief(sb + C::kDrain, 0) && globaltimer_ns() - t0 < kWaitLimitNs) {}
      }
    }
  } else if (warp < kSoftmaxWarps) {
    // ------------------------------ softmax ----------------------------------------------------
    const int side = warp / 8, half = (warp / 4) & 1, quad = warp % 4;
    const int row = quad * 32 + lane;  // of the side
    const uint32_t t_lane = tmem + ((uint32_t)(quad * 32) << 16);
    const uint32_t t_s = t_lane + side * 128 + half * 64;  // this thread's columns of S; P goes to the first 32 of them
    const uint32_t t_o = t_lane + C::kColO + side * DH + half * (DH / 2);
    float* sum_own = reinterpret_cast<float*>(smem + C::kOffSum) + (side * 2 + half) * kSide + row;  // + 4 * 128 for odd blocks
    const float* sum_other = reinterpret_cast<const float*>(smem + C::kOffSum) + (side * 2 + (half ^ 1)) * kSide + row;
    float* max_own = reinterpret_cast<float*>(smem + C::kOffMax) + (side * 2 + half) * kSide + row;
    const float* max_other = reinterpret_cast<const float*>(smem + C::kOffMax) + (side * 2 + (half ^ 1)) * kSide + row;
    float4* ends = reinterpret_cast<float4*>(smem + C::kOffEnd) + row;  // + (side * 2 + half) * 128
    uint32_t cnt_s = 0, cnt_o[2] = {0, 0}, cnt_pair = 0, cnt_quad = 0;
    auto meet = [&](bool four) {  // the warps that share these 32 rows
      __syncwarp();
      const uint32_t bar = four ? sb + C::kQuad + 8 * quad : sb + C::kPair + 8 * (side * 4 + quad);
      if (lane == 0) mbar_arrive(bar);
      const bool met = mbar_wait_paced(bar, (four ? cnt_quad : cnt_pair) & 1, abort_flag, p.status, kStatusCache | 12);
      if (four) ++cnt_quad; else ++cnt_pair;
      return __all_sync(0xffffffffu, met) != 0;
    };
    const int32_t side_rows = per_side * p.group;
    for (; walk.more(); walk.next(p, view)) {
      const AttnEntry e = view.entry[walk.entry];
      const bool split = e.count <= per_side;  // both sides on the same rows
      const int32_t tile_row = (split ? 0 : side * side_rows) + row;
      const int32_t t = (split ? 0 : side * per_side) + row / p.group, h = walk.head * p.group + row % p.group;
      const bool there = row < side_rows && t < e.count;
      RowKeys keys{0, 0, 0};
      float slope = 0.f;
      if (there) {
        keys = attn_row(p, e, t);
        if (BIAS) slope = slope_of(p, h);
      }
      const bool sees = there && keys.lo < keys.hi;
      uint8_t* out = p.O + (int64_t)(e.row0 + t) * p.o_row_bytes + h * p.o_head_bytes;
      if (e.blocks == 0) {  // nobody sees a key
        if (there && half == 0 && (!split || side == 0))
#pragma unroll
          for (int c = 0; c < DH / 8; ++c) reinterpret_cast<uint4*>(out)[c] = make_uint4(0u, 0u, 0u, 0u);
        continue;
      }
      // rows that do not exist ask for no mask
      const int32_t lo_most = __reduce_max_sync(0xffffffffu, there ? keys.lo : 0);
      const int32_t hi_least = __reduce_min_sync(0xffffffffu, there ? keys.hi : 0x7fffffff);
      const int32_t blk0 = e.blk0 + walk.block0(p), n = walk.blocks(p);
      const int32_t step = split ? 2 : 1, first = split ? side : 0;
      // -inf: no reference yet.  Capped scores need none, unless the cap is beyond what fp32's range has room for.
      const bool bounded = CAP && !BIAS && p.cap <= 80.f;
      float m = sees && !bounded ? -INFINITY : 0.f, l = 0.f;
      float own[2] = {0.f, 0.f};  // this half's sums of the last two blocks
      float moved = 1.f;          // 2^(what the reference moved by for the last block)
      bool aborted = false;
      for (int32_t i = first; i < n; i += step) {
        // The reference moves by what the block before the last one summed to: that the other half's sum of it is there is
        // known since the last block's S arrived, so that nothing of this comes behind this block's.
        float up = 0.f;
        if (i >= first + 2 * step) {
          const float most = fmaxf(own[cnt_s & 1], sum_other[((cnt_s - 2) & 3) * 4 * kSide]);
          // (as long as the reference moved for the block in front of it, its sum was that of the old one)
          // (and by what fp32 lets it: scores of 2^24 and more are further apart than 1)
          if (most > kMoveAt * moved) up = rintf((m + (float)((int32_t)(__float_as_uint(most / moved) >> 23) - 127)) - m);
        }
        const bool slow = __any_sync(0xffffffffu, m == -INFINITY || up != 0.f);
        if (!mbar_wait_suspended(sb + C::kSFull + 8 * side, cnt_s & 1, abort_flag, p.status, kStatusCache | 10)) { aborted = true; break; }
        tc_fence_after_sync();
        const int32_t b0 = (blk0 + n - 1 - i) * BK, j0 = b0 + half * 64;  // the block's first key, this thread's
        // what masks may be left out, by the keys of this half (long chunk: 492 us, by those of the whole block 504 us), or of the
        // block where scores are capped (first visits: 133.5 and 132.3 us)
        const bool all_begun = (CAP ? b0 : j0) >= lo_most, none_ended = (CAP ? b0 + BK : j0 + 64) <= hi_least;
        auto mask = [&](int c0, uint32_t (&s)[16]) {
          if (!all_begun) {
            const int32_t lo = keys.lo - j0 - c0;
#pragma unroll
            for (int x = 0; x < 16; ++x)
              if (x < lo) s[x] = 0xff800000u;
          }
          if (!none_ended) {
            const int32_t hi = keys.hi - j0 - c0;
#pragma unroll
            for (int x = 0; x < 16; ++x)
              if (x >= hi) s[x] = 0xff800000u;
          }
        };
        // scores of columns c0.. in log2 units but for a factor (`scale`), -inf where the row does not see the key
        const float scale = BIAS ? 1.f : CAP ? p.cap : p.scale;
        auto scores = [&](int c0, uint32_t (&s)[16]) {
          if (CAP) {
            float most = 0.f;
#pragma unroll
            for (int x = 0; x < 16; x += 2) {
              uint64_t u;
              float t0, t1, u0, u1;
              unpack2(tanh_pair<CAP == 1>(fmul2(pack2(__uint_as_float(s[x]), __uint_as_float(s[x + 1])), pack2(p.scale, p.scale)), u), t0, t1);
              unpack2(u, u0, u1);
              most = fmax3(most, u0, u1);
              s[x] = __float_as_uint(t0);
              s[x + 1] = __float_as_uint(t1);
            }
            const bool beyond = !(most <= kTanhRange2);
            if (__any_sync(0xffffffffu, beyond)) {  // rows with a score beyond the polynomial's range: from S again
              uint32_t again[16];
              tmem_ld_32x32b_x16(t_s + c0, again);
              tmem_ld_wait();
#pragma unroll
              for (int x = 0; x < 16; ++x) {
                const float t = CAP == 1 ? tanh_far(__uint_as_float(again[x]) * p.scale) : tanh_of(__uint_as_float(again[x]) * p.scale);
                if (beyond) s[x] = __float_as_uint(t);  // (a row's own way, whatever the others take)
              }
            }
          }
          if (BIAS) {
            const float away = (float)(keys.pos - j0 - c0), factor = CAP ? p.cap : p.scale;
#pragma unroll
            for (int x = 0; x < 16; ++x)
              s[x] = __float_as_uint(fmaf(-slope, fabsf(away - (float)x), __uint_as_float(s[x]) * factor));
          }
          mask(c0, s);
        };
        if (slow) {
          if (__any_sync(0xffffffffu, m == -INFINITY)) {  // rows without a reference: the maximum of this block
            float mx = -INFINITY;
#pragma unroll 1
            for (int c = 0; c < 64; c += 32) {
              uint32_t s[2][16];
              tmem_ld_32x32b_x16(t_s + c, s[0]);
              tmem_ld_32x32b_x16(t_s + c + 16, s[1]);
              tmem_ld_wait();
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                if (BIAS) scores(c + y * 16, s[y]); else mask(c + y * 16, s[y]);
#pragma unroll
                for (int x = 0; x < 16; x += 2) mx = fmax3(mx, __uint_as_float(s[y][x]), __uint_as_float(s[y][x + 1]));
              }
            }
            if (!BIAS) mx = !CAP ? mx * scale : mx == -INFINITY ? mx : scale * tanh_of(mx * p.scale);  // (a cap keeps the order)
            *max_own = mx;
            if (!meet(false)) { aborted = true; break; }
            if (m == -INFINITY) m = fmaxf(mx, *max_other);
          }
          if (__any_sync(0xffffffffu, up != 0.f)) {
            const float a = exp2_down((int32_t)up);
            m += up;
            l *= a;
#pragma unroll 1
            for (int c = 0; c < DH / 2; c += 16) {
              uint32_t o[16];
              tmem_ld_32x32b_x16(t_o + c, o);
              tmem_ld_wait();
#pragma unroll
              for (int x = 0; x < 16; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * a);
              tmem_st_32x32b_x16(t_o + c, o);
            }
          }
        }
        moved = __uint_as_float((uint32_t)min(127 + (int32_t)up, 254) << 23);
        const float ref = m == -INFINITY ? 0.f : m;
        const uint64_t c2 = pack2(scale, scale), m2 = pack2(-ref, -ref);
        uint64_t sum2 = pack2(0.f, 0.f);
        // 16 columns at a time, the next ones on their way (P's columns are those of scores that have been read)
        uint32_t s[2][16];
        tmem_ld_32x32b_x16(t_s, s[0]);
        tmem_ld_wait();
        // `some`: how many of eight pairs take the FMA pipes instead of the special-function unit.  With heads of 64 a block's
        // exponentials take twice as long as its products (candidates of 32 requests: 127 us without, 122 us with two of
        // eight, 128 us with four); with heads of 128 the same time (long chunk: 479 us without, 484 us with two).
        auto weights = [&](auto some) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            if (c > 0) tmem_ld_wait();
            if (c < 3) tmem_ld_32x32b_x16(t_s + (c + 1) * 16, s[(c + 1) % 2]);
            scores(c * 16, s[c % 2]);
            uint32_t pk[8];
#pragma unroll
            for (int x = 0; x < 16; x += 2) {
              const uint64_t x2 = ffma2(pack2(__uint_as_float(s[c % 2][x]), __uint_as_float(s[c % 2][x + 1])), c2, m2);
              float p0, p1;
              if ((x / 2 * 3) % 8 < decltype(some)::value) {
                unpack2(exp2_pair(x2), p0, p1);
              } else {
                float x0, x1;
                unpack2(x2, x0, x1);
                p0 = ex2_approx(x0);
                p1 = ex2_approx(x1);
              }
              sum2 = fadd2(sum2, pack2(p0, p1));
              pk[x / 2] = bf16_pair(p0, p1);
            }
            tmem_st_x8(t_s + c * 8, pk);
            if (c + 1 == kFirst) {  // the products of these keys may begin
              tmem_st_wait();
              tc_fence_before_sync();
              __syncwarp();
              if (lane == 0) mbar_arrive(sb + C::kPHalf + 8 * side);
            }
          }
        };
        // blocks without a mask on code of their own (long chunk: 531 us on one for both) where scores are not capped (first
        // visits: 175 us on one, 186 us on two)
        if (!CAP && all_begun && none_ended) weights(std::integral_constant<int, DH == 64 ? 2 : 0>());
        else weights(std::integral_constant<int, 0>());  // (a masked key's weight is 0 there, not 2^-125)
        float s0, s1;
        unpack2(sum2, s0, s1);
        own[cnt_s & 1] = sees ? s0 + s1 : 0.f;
        l += s0 + s1;
        sum_own[(cnt_s & 3) * 4 * kSide] = own[cnt_s & 1];
        ++cnt_s;
        tmem_st_wait();
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(sb + C::kPFull + 8 * side);
      }
      if (aborted) break;
      // ---- end of the piece: two (split: four) threads per row have a share of its columns each
      const bool both = split && n > 1;  // O of either side
      // Which sides' O this tile has, and which of them this thread reads.  (The arrivals of a side that it does not read are
      // counted too: side A's of a piece comes in front of side B's, and both in front of the next piece's.)
      bool done = true;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (s == 1 && split && !both) continue;
        if (split || s == side)
          done = done && mbar_wait_paced(sb + C::kOFull + 8 * s, cnt_o[s] & 1, abort_flag, p.status, kStatusCache | 11);
        ++cnt_o[s];
      }
      if (!done) break;
      tc_fence_after_sync();
      const int32_t width = split ? DH / 4 : DH / 2, col0 = (split ? side * 2 + half : half) * width;
      const uint32_t t_a = t_lane + C::kColO + (split ? 0 : side * DH) + col0, t_b = t_lane + C::kColO + DH + col0;
      // A side without a block of this piece has met nobody since the end of the piece in front, where its first half may still
      // be reading the probes of both.  (Otherwise the arrival of O, for which all warps of the side have brought P, comes behind.)
      if (first >= n && !meet(false)) break;
      ends[(side * 2 + half) * kSide] = make_float4(m, l, 0.f, 0.f);
      if (!meet(split)) break;
      float wa = 1.f, wb = 0.f, m_all = m, l_all;
      if (split) {
        const float4 a0 = ends[0], a1 = ends[kSide], b0 = ends[2 * kSide], b1 = ends[3 * kSide];
        m_all = a0.x;
        l_all = a0.y + a1.y;
        if (both) {
          m_all = fmaxf(a0.x, b0.x);
          const float r = m_all == -INFINITY ? 0.f : m_all;
          // (denormal weights count: the sums beside them may be up to 2^128)
          wa = exp2f(a0.x - r);
          wb = exp2f(b0.x - r);
          l_all = wa * l_all + wb * (b0.y + b1.y);
        }
      } else {
        l_all = ends[side * 2 * kSide].y + ends[(side * 2 + 1) * kSide].y;
      }
      const bool whole = walk.whole();
      const int32_t part = walk.part();
      float inv = whole ? (sees ? 1.f / l_all : 0.f) : 1.f;
      const bool beyond = !(l_all < INFINITY);
      if (!whole && l_all > 0x1p64f) {  // the reference is where the sum is, so that sums of parts stay in fp32's range
        const float by = rintf((m_all + (float)((int32_t)(__float_as_uint(l_all) >> 23) - 127)) - m_all);
        inv = exp2_down((int32_t)by);
        m_all += by;
        l_all *= inv;
      }
      // non-finite, or only scores of -inf, which exp2_pair does not take to 0: by hand
      float probe = m == -INFINITY && l != 0.f ? NAN : l * 0.f;
      float* to = attn_part(p, part) + (int64_t)tile_row * DH + col0;
      const uint32_t rows_there = __ballot_sync(0xffffffffu, there);
      const int lane4 = lane & 3, lane0 = lane & ~3;
      uint8_t* out4[4];  // the rows of this lane and its three neighbours
#pragma unroll
      for (int k = 0; k < 4; ++k)
        out4[k] = reinterpret_cast<uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(out), lane0 + k));
      auto column = [&](uint32_t a, uint32_t b) {  // of the row's result
        float v = __uint_as_float(a) * wa;
        if (both) v = fmaf(__uint_as_float(b), wb, v);
        probe = fmaf(v, 0.f, probe);
        return v * inv;
      };
#pragma unroll 1
      for (int c = 0; c < width; c += 16) {
        uint32_t o[16], ob[16];
        tmem_ld_32x32b_x16(t_a + c, o);
        if (both) tmem_ld_32x32b_x16(t_b + c, ob);
        tmem_ld_wait();
        uint4 v[4];
        if (whole) {  // 16 columns: two pieces, and with the next 16 of a wide share four
#pragma unroll
          for (int x = 0; x < 2; ++x)
            v[x] = make_uint4(bf16_pair(column(o[8 * x], ob[8 * x]), column(o[8 * x + 1], ob[8 * x + 1])),
                              bf16_pair(column(o[8 * x + 2], ob[8 * x + 2]), column(o[8 * x + 3], ob[8 * x + 3])),
                              bf16_pair(column(o[8 * x + 4], ob[8 * x + 4]), column(o[8 * x + 5], ob[8 * x + 5])),
                              bf16_pair(column(o[8 * x + 6], ob[8 * x + 6]), column(o[8 * x + 7], ob[8 * x + 7])));
          if (width == 16) {
            if (there) {
              *reinterpret_cast<uint4*>(out + col0 * 2) = v[0];
              *reinterpret_cast<uint4*>(out + col0 * 2 + 16) = v[1];
            }
            continue;
          }
          c += 16;
          tmem_ld_32x32b_x16(t_a + c, o);
          if (both) tmem_ld_32x32b_x16(t_b + c, ob);
          tmem_ld_wait();
#pragma unroll
          for (int x = 0; x < 2; ++x)
            v[2 + x] = make_uint4(bf16_pair(column(o[8 * x], ob[8 * x]), column(o[8 * x + 1], ob[8 * x + 1])),
                                  bf16_pair(column(o[8 * x + 2], ob[8 * x + 2]), column(o[8 * x + 3], ob[8 * x + 3])),
                                  bf16_pair(column(o[8 * x + 4], ob[8 * x + 4]), column(o[8 * x + 5], ob[8 * x + 5])),
                                  bf16_pair(column(o[8 * x + 6], ob[8 * x + 6]), column(o[8 * x + 7], ob[8 * x + 7])));
          transpose_pieces(v, lane);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if ((rows_there >> (lane0 + k)) & 1) *reinterpret_cast<uint4*>(out4[k] + (col0 + c - 16) * 2 + lane4 * 16) = v[k];
        } else {
#pragma unroll
          for (int x = 0; x < 4; ++x)
            v[x] = make_uint4(__float_as_uint(column(o[4 * x], ob[4 * x])), __float_as_uint(column(o[4 * x + 1], ob[4 * x + 1])),
                              __float_as_uint(column(o[4 * x + 2], ob[4 * x + 2])), __float_as_uint(column(o[4 * x + 3], ob[4 * x + 3])));
          transpose_pieces(v, lane);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if ((rows_there >> (lane0 + k)) & 1) *reinterpret_cast<uint4*>(to + (lane0 + k - lane) * DH + c + lane4 * 4) = v[k];
        }
      }
      const bool leads = half == 0 && (!split || side == 0);  // of the threads of a row
      if (there && !whole && leads) attn_part_sums(p, gridDim.x, part)[tile_row] = make_float2(m_all, l_all);
      ends[(side * 2 + half) * kSide].z = probe;
      tc_fence_before_sync();  // the next piece's first P V overwrites O
      if (!meet(split)) break;  // O has been read, and what there is of a row written
      bool bad = false;
      if (leads) {
        bad = there && (split ? ends[0].z + ends[kSide].z + ends[2 * kSide].z + ends[3 * kSide].z
                              : ends[side * 2 * kSide].z + ends[(side * 2 + 1) * kSide].z) != 0.f;
        bad = bad || (there && beyond);
        // Scores of 2^30 and more: their product with the scale is not rounded where the reference was, so that the largest weight
        // may have come out as 2^-64 and less, beside others that 2^-126 or exp2_pair's least cut off.  (Without a reference it may
        // be 2^-80.)
        bad = bad || (sees && l_all < (bounded ? 0x1p-100f : 0x1p-64f) && keys.lo < (blk0 + n) * BK && keys.hi > blk0 * BK);
      }
      uint32_t redo = __ballot_sync(0xffffffffu, bad);
      while (redo != 0) {  // a row at a time, by the warp
        const int src = __ffs(redo) - 1;
        redo &= redo - 1;
        const int32_t r = quad * 32 + src, rt = (split ? 0 : side * per_side) + r / p.group, rh = walk.head * p.group + r % p.group;
        const RowKeys rk = attn_row(p, e, rt);
        float acc[DH / 32], mm, ll;
        attn_row_by_hand<DH>(p, e, (int64_t)(walk.head / p.per_kv) * p.head_bytes,
                             p.Q + (int64_t)(e.row0 + rt) * p.q_row_bytes + rh * p.q_head_bytes, rk, slope_of(p, rh), blk0 * BK,
                             (blk0 + n) * BK, mm, ll, acc);
        if (whole) {
          __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(p.O + (int64_t)(e.row0 + rt) * p.o_row_bytes + rh * p.o_head_bytes);
#pragma unroll
          for (int c = 0; c < DH / 32; ++c) o[lane + 32 * c] = __float2bfloat16_rn(rk.lo < rk.hi ? acc[c] / ll : 0.f);
        } else {
          const int32_t tr = (split ? 0 : side * side_rows) + r;
          float* o = attn_part(p, part) + (int64_t)tr * DH;
#pragma unroll
          for (int c = 0; c < DH / 32; ++c) o[lane + 32 * c] = acc[c];
          if (lane == 0) attn_part_sums(p, gridDim.x, part)[tr] = make_float2(mm, ll);
        }
      }
    }
  }

  tc_fence_before_sync();
  __syncthreads();
  if (warp == kIssue) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

template <int DH, int CAP, bool BIAS>
rocs_status_t launch_umma(const CacheAttn& p, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, int32_t grid,
                          cudaStream_t stream) {
  auto kernel = umma_kernel<DH, CAP, BIAS>;
  ROCS_ALLOW_SMEM(kernel, UmmaCfg<DH>::kSmem);
  return launch_dependent(kernel, dim3((unsigned)grid), kUmmaThreads, (size_t)UmmaCfg<DH>::kSmem, stream, q, k, v, p);
}
template <int DH>
rocs_status_t umma_of(const CacheAttn& p, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, int32_t grid,
                      cudaStream_t stream) {
  const int cap = !(p.cap > 0.f) ? 0 : p.cap <= kShortCap * 1.4426950408889634f ? 1 : 2;  // (p.cap is in log2 units)
  if (cap == 2) return p.slopes ? launch_umma<DH, 2, true>(p, q, k, v, grid, stream) : launch_umma<DH, 2, false>(p, q, k, v, grid, stream);
  if (cap == 1) return p.slopes ? launch_umma<DH, 1, true>(p, q, k, v, grid, stream) : launch_umma<DH, 1, false>(p, q, k, v, grid, stream);
  return p.slopes ? launch_umma<DH, 0, true>(p, q, k, v, grid, stream) : launch_umma<DH, 0, false>(p, q, k, v, grid, stream);
}

}  // namespace

bool attn_umma_supported(int32_t dh, int32_t page) {
  return (dh == 64 || dh == 128) && (page % BK == 0 || page == 64 || page == 32 || page == 16 || page == 8);
}

rocs_status_t attn_umma(const CacheAttn& p, int32_t H, int32_t H_kv, int64_t N, int32_t grid, cudaStream_t stream) {
  // a dimension of one entry keeps a stride that a tensor map takes
  const uint64_t dh = (uint64_t)p.dh, dense = dh * 2;
  auto stride = [&](int64_t bytes) { return bytes > 0 ? (uint64_t)bytes : dense; };
  CUtensorMap q, k, v;
  const uint64_t q_dims[3] = {dh, (uint64_t)H, (uint64_t)N}, q_strides[2] = {stride(H > 1 ? p.q_head_bytes : 0), stride(N > 1 ? p.q_row_bytes : 0)};
  const uint32_t q_box[3] = {64, (uint32_t)p.group, (uint32_t)(p.rows_per_tile / 2)};
  if (!make_tensor_map_bf16(&q, p.Q, 3, q_dims, q_strides, q_box) || !make_page_map(&k, p.K, p, H_kv, BK) ||
      !make_page_map(&v, p.V, p, H_kv, BK))
    return ROCS_ERR_CUDA;
  return p.dh == 128 ? umma_of<128>(p, q, k, v, grid, stream) : umma_of<64>(p, q, k, v, grid, stream);
}

}  // namespace rocs
