// Attention over a paged cache for many rows of a (sequence, KV head): slots of
// 128 rows on tcgen05, two of them sharing every K/V tile that the CTA loads.
// A persistent CTA per SM walks its even share of all units (128 keys of a row
// tile); every role runs on across the borders of problems.
//   warps 0-3, 4-7  softmax of slot 0, 1: a thread per row (TMEM lane), with the
//                   running max, row sum and the rescale of O in TMEM; at a
//                   segment's end the slot's fp32 partial
//   warp 8          K pages by TMA into a 3-deep ring (128B swizzle)
//   warp 9          S = Q K^T and O += P V (A = P from TMEM, over S)
//   warp 10         V pages into a 2-deep ring
//   warp 11         Q of the segment's slots, by a map whose box is the group's
//                   heads of as many tokens as 128 rows hold
// Per key tile: P0.V, S0 of the next tile, P1.V, S1 of the next tile, so that the
// tensor pipe works on one slot while the softmax works on the other. With one
// slot the other slot's S columns are a second S buffer.
// A thread holds no row of S across its two passes (maximum, then P): in registers
// it took as long. The running max moves only when it grows by more than 2^8; P is
// rounded to 16 bits for its product with V (the MMA's operand type), its sum is not.
// A slot's chain is the bound, S -> softmax (about 2,000 clocks) -> P.V and the
// next S: 3,300 clocks a tile of two slots against 2,560 of tensor pipe. 64-token trees over
// four caches of 65,664 tokens, 7 heads a KV head of 128: 215 us from a cold L2, 1,115 TFLOP/s, the
// tensor pipe 58% busy.
#include <cstdint>
#include <cuda_runtime.h>

#include "cache_attn.cuh"

namespace evisel {
namespace {

constexpr int kRows = 128;
constexpr int kKeys = 128;
constexpr int kWarpK = 8, kWarpMma = 9, kWarpV = 10, kWarpQ = 11;
constexpr int kThreads = 384;
constexpr int NK = 3, NV = 2;

template <int D>
struct WideCfg {
  static constexpr int KB = D / 64;
  static constexpr int BLOCK = kKeys * 128;      // a 64-column block of 128 rows
  static constexpr int TILE = KB * BLOCK;
  static constexpr int OFF_Q = 0;                // two slots
  static constexpr int OFF_K = 2 * TILE;
  static constexpr int OFF_V = OFF_K + NK * TILE;
  static constexpr int OFF_BAR = OFF_V + NV * TILE;
  static constexpr int B_QF = 0, B_QE = 1;       // the segment's Q: landed, read by its last S
  static constexpr int B_KF = 2, B_KE = B_KF + NK, B_VF = B_KE + NK, B_VE = B_VF + NV;
  // S computed: slot 0's, slot 1's, and the second buffer's where there is one slot. Each has one group of waiters,
  // which waits for every phase: a group that skipped some could take an older phase of the same parity for its own.
  static constexpr int B_SF = B_VE + NV;
  static constexpr int B_PF = B_SF + 3;          // 2 S buffers: P written (128 arrivals)
  static constexpr int B_OF = B_PF + 2;          // 2 slots: O complete
  static constexpr int B_DRAIN = B_OF + 2;
  static constexpr int N_BARS = B_DRAIN + 1;
  static constexpr int OFF_MISC = OFF_BAR + N_BARS * 8;   // TMEM address, abort flag, split scratch
  static constexpr int SMEM_USED = OFF_MISC + 8 + 40 * 4 + 1024;
  static constexpr int SMEM = SMEM_USED < 120 * 1024 ? 120 * 1024 : SMEM_USED;   // one CTA per SM: TMEM is taken whole
  static constexpr int COL_O = 128;              // per slot: S (128 columns) | O (D)
  static constexpr int SLOT_COLS = 128 + D;
  static_assert(SMEM <= 232448, "shared memory budget");
};

template <class T>
constexpr uint32_t idesc(int M, int N, bool b_mn) {
  return (1u << 4) | (T::kFormat << 7) | (T::kFormat << 10) | ((b_mn ? 1u : 0u) << 16) |
         (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}

// Slots of a segment that hold rows.
__device__ __forceinline__ int slots_of(const CacheAttnLaunch& L, const Segment& s) {
  const int left = L.rows - s.rt * L.slots * L.slot_rows;
  return L.slots == 2 && left > L.slot_rows ? 2 : 1;
}

// Pages of K or V: lane i sends box i of a tile.
template <int D, bool IS_V>
__device__ __forceinline__ void load_pages(const CacheAttnLaunch& L, const UnitCount& uc, Walk walk, uint32_t sbase,
                                           volatile int* abort_flag) {
  using C = WideCfg<D>;
  auto bar = [&](int i) { return sbase + C::OFF_BAR + 8u * i; };
  constexpr int R = IS_V ? NV : NK, FULL = IS_V ? C::B_VF : C::B_KF, EMPTY = IS_V ? C::B_VE : C::B_KE;
  const CUtensorMap* map = IS_V ? &L.tm_v : &L.tm_k;
  const int perm = IS_V ? L.v_perm : L.k_perm;
  const int lane = threadIdx.x & 31, kb = lane % C::KB, sub = lane / C::KB, subs = kKeys / L.box_rows;
  const uint64_t pol = ptx::l2_policy_evict_first();
  Segment s;
  uint32_t n = 0;
  bool ok = true;
  while (ok && walk.next(L.c, L.row_tiles, uc, s, L.status)) {
    for (int t = s.t0; t < s.t1; ++t, ++n) {
      const int st = n % R, key0 = t * kKeys + sub * L.box_rows;
      const bool mine = sub < subs && key0 < s.len;
      const int id = mine ? cache_page(L.c, s.b, s.h, key0 >> L.c.log_page, L.status) : 0;
      if (n >= R && !warp_wait(bar(EMPTY + st), (n / R - 1) & 1, abort_flag)) {
        ok = false;
        break;
      }
      const int boxes = min(subs, (s.len - t * kKeys + L.box_rows - 1) / L.box_rows) * C::KB;
      if (lane == 0) ptx::mbar_arrive_expect_tx(bar(FULL + st), boxes * L.box_rows * 128);
      __syncwarp();
      if (mine)
        ptx::tma_load_page(sbase + (IS_V ? C::OFF_V : C::OFF_K) + st * C::TILE + kb * C::BLOCK + sub * L.box_rows * 128,
                           map, bar(FULL + st), perm, kb * 64, key0 & (L.c.page - 1), s.h, id, pol);
    }
  }
  if (!ok && lane == 0) record_timeout(abort_flag, L.status);
  const volatile int never = 0;                  // no copy in flight at exit
  for (uint32_t i = 0; i < R && i < n; ++i)
    ptx::mbar_wait(bar(FULL + (n - 1 - i) % R), ((n - 1 - i) / R) & 1, &never, kWaitTimeoutNs);
}

template <int D>
__device__ __forceinline__ void load_queries(const CacheAttnLaunch& L, const UnitCount& uc, Walk walk, uint32_t sbase,
                                             volatile int* abort_flag) {
  using C = WideCfg<D>;
  auto bar = [&](int i) { return sbase + C::OFF_BAR + 8u * i; };
  const int lane = threadIdx.x & 31, tokens = L.qt.tokens;         // of a slot
  const uint64_t pol = ptx::l2_policy_evict_last();
  Segment s;
  uint32_t n = 0;                                // segments
  bool ok = true;
  for (; ok && walk.next(L.c, L.row_tiles, uc, s, L.status); ++n) {
    if (n >= 1 && !warp_wait(bar(C::B_QE), (n - 1) & 1, abort_flag)) {
      ok = false;
      break;
    }
    const int ns = slots_of(L, s);
    if (lane == 0) {
      ptx::mbar_arrive_expect_tx(bar(C::B_QF), ns * C::KB * L.slot_rows * 128);
      for (int i = 0; i < ns; ++i)
        for (int kb = 0; kb < C::KB; ++kb)
          ptx::tma_load_page(sbase + C::OFF_Q + i * C::TILE + kb * C::BLOCK, &L.tm_q, bar(C::B_QF), L.q_perm, kb * 64,
                             (s.rt * L.slots + i) * tokens, s.h * L.d.gq, s.b, pol);
    }
    __syncwarp();
  }
  if (!ok && lane == 0) record_timeout(abort_flag, L.status);
  const volatile int never = 0;
  if (n > 0) ptx::mbar_wait(bar(C::B_QF), (n - 1) & 1, &never, kWaitTimeoutNs);
}

// The whole warp walks the tiles; one elected lane issues every MMA and commit
// (tcgen05.commit tracks the MMAs of the thread that issues it, so the lane
// must not change; a change is treated as a failure).
template <class T, int D>
__device__ __forceinline__ void issue_mmas(const CacheAttnLaunch& L, const UnitCount& uc, Walk walk, uint32_t sbase_in,
                                           uint32_t tmem_in, volatile int* abort_flag) {
  using C = WideCfg<D>;
  const uint32_t sbase = __shfl_sync(0xffffffffu, sbase_in, 0);
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_in, 0);
  auto bar = [&](int i) { return sbase + C::OFF_BAR + 8u * i; };
  constexpr uint32_t kIdescS = idesc<T>(kRows, kKeys, false), kIdescO = idesc<T>(kRows, D, true);
  const int lane = threadIdx.x & 31;
  uint32_t leader = 0;
  int first_leader = -1;
  bool same = true, issued = false, ok = true;
  auto elect = [&]() -> bool {
    const bool me = ptx::elect_one(leader);
    if (first_leader < 0) first_leader = static_cast<int>(leader);
    same = same && static_cast<int>(leader) == first_leader;
    return me && same;
  };
  const uint64_t dq = ptx::sdesc_sw128(sbase + C::OFF_Q, 16, 1024);
  const uint64_t dk = ptx::sdesc_sw128(sbase + C::OFF_K, 16, 1024);
  const uint64_t dv = ptx::sdesc_sw128(sbase + C::OFF_V, C::BLOCK, 1024);
  auto mma_s = [&](int slot, uint32_t n, int buf) {
    const uint64_t qd = dq + static_cast<uint64_t>(slot * C::TILE >> 4);
    const uint64_t kd = dk + static_cast<uint64_t>((n % NK) * C::TILE >> 4);
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      const uint64_t off = static_cast<uint64_t>(((kk / 4) * C::BLOCK + (kk % 4) * 32) >> 4);
      ptx::mma_ss(tmem + buf * C::SLOT_COLS, qd + off, kd + off, kIdescS, kk > 0 ? 1u : 0u);
    }
  };
  // O_slot (+)= P V over the tile's first `ksteps` groups of 16 keys, P from S[buf].
  auto mma_pv = [&](int slot, uint32_t n, int buf, int ksteps, bool add) {
    const uint64_t vd = dv + static_cast<uint64_t>((n % NV) * C::TILE >> 4);
#pragma unroll
    for (int kk = 0; kk < kKeys / 16; ++kk)
      if (kk < ksteps)
        ptx::mma_ts(tmem + slot * C::SLOT_COLS + C::COL_O, tmem + buf * C::SLOT_COLS + kk * 8,
                    vd + static_cast<uint64_t>((kk * 16 * 128) >> 4), kIdescO, add || kk > 0 ? 1u : 0u);
  };
  // A tile that reaches past the sequence's end: the values of its last group of
  // 16 past the end may be anything, so they are zeroed (once, after it landed).
  auto zero_tail = [&](uint32_t n, int left) {
    const int row0 = left, rows = ((left + 15) & ~15) - left;
    for (int i = lane; i < rows * C::KB * 8; i += 32) {
      const int row = row0 + i / (C::KB * 8), x = i % (C::KB * 8);
      asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(sbase + C::OFF_V + (n % NV) * C::TILE +
                                                                    (x / 8) * C::BLOCK + row * 128 + (x % 8) * 16),
                   "r"(0)
                   : "memory");
    }
    ptx::fence_proxy_async_smem();
    __syncwarp();
  };

  Segment s;
  uint32_t n = 0, seg = 0, pf = 0;               // tiles and segments so far; parity of the P waits, a bit per buffer
  while (ok && walk.next(L.c, L.row_tiles, uc, s, L.status)) {
    const bool two = slots_of(L, s) == 2;
    const int cnt = s.t1 - s.t0;
    ok = warp_wait(bar(C::B_QF), seg & 1, abort_flag) && warp_wait(bar(C::B_KF + n % NK), (n / NK) & 1, abort_flag);
    if (!ok) break;
    // The first S of the segment (with one slot the first two: the buffers alternate).
    ptx::tc_fence_after();
    if (elect()) {
      mma_s(0, n, 0);
      ptx::mma_commit(bar(C::B_SF));
      if (two) {
        mma_s(1, n, 1);
        ptx::mma_commit(bar(C::B_SF + 1));
      }
      ptx::mma_commit(bar(C::B_KE + n % NK));
      if (cnt == 1) ptx::mma_commit(bar(C::B_QE));
    }
    __syncwarp();
    issued = true;
    ok = same;
    if (ok && !two && cnt > 1) {
      ok = warp_wait(bar(C::B_KF + (n + 1) % NK), ((n + 1) / NK) & 1, abort_flag);
      if (!ok) break;
      if (elect()) {
        mma_s(0, n + 1, 1);
        ptx::mma_commit(bar(C::B_SF + 2));
        ptx::mma_commit(bar(C::B_KE + (n + 1) % NK));
        if (cnt == 2) ptx::mma_commit(bar(C::B_QE));
      }
      __syncwarp();
      ok = same;
    }
    const int ahead = two ? 1 : 2;               // S runs this many tiles ahead of P.V
    for (int j = 0; ok && j < cnt; ++j, ++n) {
      const int left = s.len - (s.t0 + j) * kKeys, ksteps = left >= kKeys ? kKeys / 16 : (left + 15) / 16;
      const bool more = j + ahead < cnt, last = j + 1 == cnt;
      const uint32_t nn = n + ahead;
      ok = warp_wait(bar(C::B_VF + n % NV), (n / NV) & 1, abort_flag) &&
           (!more || warp_wait(bar(C::B_KF + nn % NK), (nn / NK) & 1, abort_flag));
      if (!ok) break;
      if (left < kKeys) zero_tail(n, left);
      for (int slot = 0; ok && slot < (two ? 2 : 1); ++slot) {
        const int buf = two ? slot : j & 1;
        ok = warp_wait(bar(C::B_PF + buf), (pf >> buf) & 1, abort_flag);
        if (!ok) break;
        pf ^= 1u << buf;
        ptx::tc_fence_after();
        if (elect()) {
          mma_pv(slot, n, buf, ksteps, j > 0);
          if (last) ptx::mma_commit(bar(C::B_OF + slot));
          if (!two || slot == 1) ptx::mma_commit(bar(C::B_VE + n % NV));
          if (more) {
            mma_s(slot, nn, buf);
            ptx::mma_commit(bar(C::B_SF + (two || buf == 0 ? buf : 2)));
            if (!two || slot == 1) {
              ptx::mma_commit(bar(C::B_KE + nn % NK));
              if (j + ahead + 1 == cnt) ptx::mma_commit(bar(C::B_QE));
            }
          }
        }
        __syncwarp();
        ok = same;
      }
    }
    ++seg;
  }
  if (!ok) {
    if (lane == 0) record_timeout(abort_flag, L.status);
    if (issued && lane == first_leader) {        // every MMA ends before TMEM is released
      const volatile int never = 0;
      ptx::mma_commit(bar(C::B_DRAIN));
      ptx::mbar_wait(bar(C::B_DRAIN), 0, &never, kWaitTimeoutNs);
    }
  }
  __syncwarp();
}

template <class T, int D>
__device__ __forceinline__ void softmax_rows(const CacheAttnLaunch& L, const UnitCount& uc, Walk walk, int slot,
                                             uint32_t sbase, uint32_t tmem_base, volatile int* abort_flag) {
  using C = WideCfg<D>;
  auto bar = [&](int i) { return sbase + C::OFF_BAR + 8u * i; };
  const int row = threadIdx.x & 127;             // TMEM lane
  const uint32_t lane_base = static_cast<uint32_t>((row >> 5) * 32) << 16;
  const uint32_t tO = tmem_base + lane_base + slot * C::SLOT_COLS + C::COL_O;
  const uint64_t scale2 = ptx::f2(L.d.scale_log2, L.d.scale_log2);
  Segment s;
  uint32_t n = 0, sf = 0, of = 0;                // tiles so far; parity of the S waits, a bit per barrier; O waits
  bool ok = true;
  while (ok && walk.next(L.c, L.row_tiles, uc, s, L.status)) {
    const bool two = slots_of(L, s) == 2;
    const int cnt = s.t1 - s.t0;
    if (slot == 1 && !two) {                     // the other slot's S takes both buffers
      n += cnt;
      continue;
    }
    float m = -INFINITY, l = 0.f;                // running max (log2 units, less the headroom), row sum
    for (int j = 0; j < cnt; ++j, ++n) {
      const int b = two ? slot : j & 1;
      const int sb = two || b == 0 ? b : 2;
      const uint32_t tS = tmem_base + lane_base + b * C::SLOT_COLS;
      ok = warp_wait(bar(C::B_SF + sb), (sf >> sb) & 1, abort_flag);
      if (!ok) break;
      sf ^= 1u << sb;
      ptx::tc_fence_after();
      const int limit = s.len - (s.t0 + j) * kKeys;              // keys from here on do not exist
      float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      uint32_t ra[32], rb[32];
      auto mask32 = [&](uint32_t (&r)[32], int c0) {
        if (limit < kKeys) {
#pragma unroll
          for (int c = 0; c < 32; ++c)
            if (c0 + c >= limit) r[c] = 0xff800000u;             // -inf
        }
      };
      auto max32 = [&](const uint32_t (&r)[32]) {
#pragma unroll
        for (int c = 0; c < 32; c += 8)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            m4[e] = ptx::max3(m4[e], __uint_as_float(r[c + 2 * e]), __uint_as_float(r[c + 2 * e + 1]));
      };
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        ptx::tmem_ld32(tS + h * 64, ra);
        ptx::tmem_ld32(tS + h * 64 + 32, rb);
        ptx::tmem_wait_ld();
        mask32(ra, h * 64);
        max32(ra);
        mask32(rb, h * 64 + 32);
        max32(rb);
      }
      const float tm = fmaf(fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])), L.d.scale_log2, -T::kHeadroom);
      const bool need = tm > m + kRescaleThreshold;
      if (__any_sync(0xffffffffu, need)) {
        const float alpha = need ? ptx::ex2(m - tm) : 1.f;
        l *= alpha;
        m = need ? tm : m;
        if (j > 0) {
          // With two slots S_j was issued after P_{j-1}.V, which has completed
          // with it; with one slot it is waited for (its V-empty barrier).
          if (!two) {
            ok = warp_wait(bar(C::B_VE + (n - 1) % NV), ((n - 1) / NV) & 1, abort_flag);
            if (!ok) break;
            ptx::tc_fence_after();
          }
#pragma unroll 1
          for (int c = 0; c < D / 16; ++c) {
            uint32_t o[16];
            ptx::tmem_ld16(tO + c * 16, o);
            ptx::tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
            ptx::tmem_st16(tO + c * 16, o);
          }
        }
      }
      const float ms = m == -INFINITY ? 0.f : m;
      const uint64_t negm2 = ptx::f2(-ms, -ms);
      uint64_t l2[4] = {0, 0, 0, 0};
      auto p32 = [&](const uint32_t (&r)[32], uint32_t (&pk)[16]) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float x0, x1;
          ptx::unf2(ptx::fma2(ptx::f2(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1])), scale2, negm2), x0, x1);
          const float p0 = ptx::ex2(x0), p1 = ptx::ex2(x1);
          l2[e & 3] = ptx::add2(l2[e & 3], ptx::f2(p0, p1));
          pk[e] = T::pack(p0, p1);
        }
      };
      // P over the first half of S, 32 columns at a time: what it overwrites has been read.
      uint32_t pk[16];
      ptx::tmem_ld32(tS, ra);
      ptx::tmem_wait_ld();
#pragma unroll
      for (int h = 0; h < 4; h += 2) {
        ptx::tmem_ld32(tS + h * 32 + 32, rb);
        mask32(ra, h * 32);
        p32(ra, pk);
        ptx::tmem_wait_ld();
        ptx::tmem_st16(tS + h * 16, pk);
        if (h == 0) ptx::tmem_ld32(tS + 64, ra);
        mask32(rb, h * 32 + 32);
        p32(rb, pk);
        if (h == 0) ptx::tmem_wait_ld();
        ptx::tmem_st16(tS + h * 16 + 16, pk);
      }
      float a0, a1, b0, b1;
      ptx::unf2(ptx::add2(l2[0], l2[1]), a0, a1);
      ptx::unf2(ptx::add2(l2[2], l2[3]), b0, b1);
      l += (a0 + a1) + (b0 + b1);
      ptx::tmem_wait_st();
      ptx::tc_fence_before();
      ptx::mbar_arrive(bar(C::B_PF + b));
    }
    ok = ok && warp_wait(bar(C::B_OF + slot), of & 1, abort_flag);
    ++of;
    if (!ok) break;
    ptx::tc_fence_after();
    const int64_t at = (static_cast<int64_t>(blockIdx.x) + s.problem) * L.tile_rows + slot * kRows + row;
    const int token = (s.rt * L.slots + slot) * L.qt.tokens + (L.qt.head_inner ? row / L.d.gq : row % L.qt.tokens);
    const bool live = row < L.slot_rows && token < L.d.tokens;
    float4* dst = reinterpret_cast<float4*>(L.part_o + at * D);
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      uint32_t r[32];
      ptx::tmem_ld32(tO + c * 32, r);
      ptx::tmem_wait_ld();
      if (live) {
#pragma unroll
        for (int q = 0; q < 8; ++q)
          dst[c * 8 + q] = make_float4(__uint_as_float(r[4 * q]), __uint_as_float(r[4 * q + 1]),
                                       __uint_as_float(r[4 * q + 2]), __uint_as_float(r[4 * q + 3]));
      }
    }
    ptx::tc_fence_before();
    if (live) L.part_ml[at] = make_float2(m, l);
  }
  if (!ok) record_timeout(abort_flag, L.status);
}

template <class T, int D>
__global__ void __launch_bounds__(kThreads, 1) cache_attn_wide_kernel(const __grid_constant__ CacheAttnLaunch L) {
  using C = WideCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t sbase = ptx::smem_addr(smem);
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::OFF_MISC + 4);
  int* scratch = reinterpret_cast<int*>(smem + C::OFF_MISC + 8);
  const int warp = threadIdx.x >> 5;

  if (threadIdx.x == 0 && L.c.max_pages > 0) {   // (without any page there is no map)
    ptx::tma_prefetch_desc(&L.tm_k);
    ptx::tma_prefetch_desc(&L.tm_v);
    ptx::tma_prefetch_desc(&L.tm_q);
  }
  ptx::grid_wait();
  ptx::grid_launch_next();
  const UnitCount uc(L.c, kKeys, L.lead, L.row_tiles, L.status);
  int ctas = 1, begin = 0, end = 0;
  const Split sp = split_find_unit(uc, scratch, [&](int total) {
    ctas = split_ctas(total, L.n_ctas, L.min_units, L.c.batch * L.c.hkv * L.row_tiles);
    const int i = blockIdx.x;
    begin = i < ctas ? split_begin(i, total, ctas) : total;
    end = i < ctas ? split_begin(i + 1, total, ctas) : total;
    return begin;
  });
  if (begin >= end) return;                      // (the whole block, before anything is started)
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::N_BARS; ++i) ptx::mbar_init(sbase + C::OFF_BAR + 8u * i, i == C::B_PF || i == C::B_PF + 1 ? kRows : 1u);
    *abort_flag = 0;
    ptx::fence_mbar_init();
  }
  // Rows of a slot past slot_rows are never loaded: zeros once and for all.
  for (int i = threadIdx.x; i < 2 * C::TILE / 16; i += kThreads) reinterpret_cast<uint4*>(smem + C::OFF_Q)[i] = make_uint4(0, 0, 0, 0);
  ptx::fence_proxy_async_smem();
  if (warp == 0) {
    ptx::tmem_alloc<512>(sbase + C::OFF_MISC);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const Walk walk{begin, end, sp.entry, sp.first};
  if (warp < 8) softmax_rows<T, D>(L, uc, walk, warp >> 2, sbase, tmem, abort_flag);
  else if (warp == kWarpK) load_pages<D, false>(L, uc, walk, sbase, abort_flag);
  else if (warp == kWarpV) load_pages<D, true>(L, uc, walk, sbase, abort_flag);
  else if (warp == kWarpQ) load_queries<D>(L, uc, walk, sbase, abort_flag);
  else issue_mmas<T, D>(L, uc, walk, sbase, tmem, abort_flag);
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc<512>(tmem);
  }
}

template <class T, int D>
cudaError_t launch_d(const CacheAttnLaunch& L, cudaStream_t stream) {
  using C = WideCfg<D>;
  auto kern = cache_attn_wide_kernel<T, D>;
  static PerDeviceAttr once;
  const cudaError_t e = raise_smem_limit(once, reinterpret_cast<const void*>(kern), C::SMEM);
  if (e != cudaSuccess) return e;
  return launch_after(kern, dim3(L.n_ctas), kThreads, C::SMEM, stream, L);
}

}  // namespace

cudaError_t launch_cache_attn_wide(const CacheAttnLaunch& L, cudaStream_t stream) {
  if (L.c.dtype == 0) return L.c.head_dim == 128 ? launch_d<BF16, 128>(L, stream) : launch_d<BF16, 64>(L, stream);
  return L.c.head_dim == 128 ? launch_d<FP16, 128>(L, stream) : launch_d<FP16, 64>(L, stream);
}

}  // namespace evisel
