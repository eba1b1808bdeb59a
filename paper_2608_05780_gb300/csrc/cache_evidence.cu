// Attention weight per cached token:
//   acc[b, h, m] (+)= sum_{t used} sum_{heads g of group h} exp(scale q . k_m - LSE).
//
// S^T = K Q^T on tcgen05 with the keys as the 128 TMEM lanes and the rows as
// columns, so that a thread adds one key's columns and nothing crosses lanes.
// A persistent CTA per SM walks its even share of the units (128 keys of a
// sequence and KV head), four at a time:
//   warps 0-15  four groups of 128 threads, a key each; the CTA's n-th unit is
//               in K stage n % 4, S buffer n % 4 and goes to group n % 4
//   warp 16     K pages by TMA, four stages
//   warp 17     the queries' tiles (up to 128 rows), three stages, read once per
//               four units, each with its rows' -LSE log2e
//   warps 18-19 the MMAs: tile by tile, for each the four units, every other one
//               each (issuing blocks while the tensor pipe is busy: one warp's
//               waits fall into the other's products)
// Few rows (decoding) leave the K stream as the bound: one token of 16 sequences, 168 MB
// in 29.6 us, 84% of a plain copy's rate. With many a tile's 128 x 128 products and
// exponentials are, and a query tile loaded once per four units keeps its traffic
// (32 KB for four products) out of the way: 128 tokens of 7 heads over 65,536 keys take 66 us, where
// the products alone need 32; a group's step is 2,200 clocks of exponentials and 1,600 until
// its next products, and four buffers of S fill the TMEM.
#include <cstdint>
#include <cuda_runtime.h>

#include "cache_attn.cuh"

namespace evisel {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kKeys = 128;
constexpr int kGroups = 4;
constexpr int kKeyWarps = kGroups * 4;
constexpr int kWarpK = kKeyWarps, kWarpQ = kWarpK + 1, kWarpMma = kWarpK + 2;
constexpr int kMmaWarps = 2;
constexpr int kThreads = 32 * (kKeyWarps + 2 + kMmaWarps);
constexpr int QS = 3;

template <int D>
struct EvCfg {
  static constexpr int KB = D / 64;
  static constexpr int BLOCK = kKeys * 128;
  static constexpr int TILE = KB * BLOCK;
  static constexpr int OFF_K = 0;
  static constexpr int OFF_Q = kGroups * TILE;
  static constexpr int OFF_LSE = OFF_Q + QS * TILE;          // [QS][128] fp32
  static constexpr int OFF_BAR = OFF_LSE + QS * 128 * 4;
  static constexpr int B_KF = 0, B_KE = B_KF + kGroups, B_QF = B_KE + kGroups, B_QE = B_QF + QS, B_SF = B_QE + QS,
                       B_SE = B_SF + kGroups, B_DRAIN = B_SE + kGroups, B_QL = B_DRAIN + kMmaWarps, N_BARS = B_QL + QS;
  static constexpr int OFF_MISC = OFF_BAR + N_BARS * 8;      // TMEM address, abort flag, split scratch
  static constexpr int SMEM_USED = OFF_MISC + 8 + 40 * 4 + 1024;
  static constexpr int SMEM = SMEM_USED < 120 * 1024 ? 120 * 1024 : SMEM_USED;   // one CTA per SM: TMEM is taken whole
  static_assert(SMEM <= 232448, "shared memory budget");
};

// One key's sum over the rows that count, from global memory. A zeroed row's
// product with a non-finite key is NaN, so that a sum that came out NaN is formed
// again here; and all of them where no TMA map can describe the queries.
template <class T, int D>
__device__ __noinline__ float counted_sum(const CacheEvidenceLaunch& L, int b, int h, int key) {
  const int64_t id = cache_page(L.c, b, h, key >> L.c.log_page, L.status);
  const uint4* k = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(L.c.k) + id * L.c.ks[0] + h * L.c.ks[1] +
                                                  (key & (L.c.page - 1)) * L.c.ks[2]);
  const int drafted = drafted_tokens(L.d, b);
  float sum = 0.f;
  for (int t = 0; t < drafted; ++t) {
    if (L.use && !__ldg(L.use + static_cast<int64_t>(b) * L.d.tokens + t)) continue;
    for (int g = 0; g < L.d.gq && !isnan(sum); ++g) {
      const int head = h * L.d.gq + g;
      const float lse = __ldg(L.lse + (static_cast<int64_t>(head) * L.c.batch + b) * L.d.tokens + t);
      if (lse == -INFINITY) continue;
      const uint4* q = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(L.d.q) + b * L.d.qs[0] +
                                                      t * L.d.qs[1] + head * L.d.qs[2]);
      float s = 0.f;
      for (int i = 0; i < D / 8; ++i) {
        float x[8], y[8];
        unpack8<T>(__ldg(k + i), x);
        unpack8<T>(__ldg(q + i), y);
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(x[e], y[e], s);
      }
      sum += ptx::ex2(fmaf(s, L.d.scale_log2, -kLog2e * lse));
    }
  }
  return sum;
}

template <class T, int D>
__global__ void __launch_bounds__(kThreads, 1) cache_evidence_kernel(const __grid_constant__ CacheEvidenceLaunch L) {
  using C = EvCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t sbase = ptx::smem_addr(smem);
  auto bar = [&](int i) { return sbase + C::OFF_BAR + 8u * i; };
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + C::OFF_MISC);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::OFF_MISC + 4);
  int* scratch = reinterpret_cast<int*>(smem + C::OFF_MISC + 8);
  float* lse_s = reinterpret_cast<float*>(smem + C::OFF_LSE);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    ptx::tma_prefetch_desc(&L.tm_k);
    ptx::tma_prefetch_desc(&L.tm_q);
  }
  ptx::grid_wait();
  ptx::grid_launch_next();
  const UnitCount uc(L.c, kKeys, 0, 1, L.status);
  int begin = 0, end = 0;
  const Split sp = split_find_unit(uc, scratch, [&](int total) {
    const int ctas = split_ctas(total, L.n_ctas, 1, L.c.batch * L.c.hkv), i = blockIdx.x;
    begin = i < ctas ? split_begin(i, total, ctas) : total;
    end = i < ctas ? split_begin(i + 1, total, ctas) : total;
    return begin;
  });
  if (begin >= end) return;                      // (the whole block, before anything is started)
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::N_BARS; ++i)
      ptx::mbar_init(bar(i), i >= C::B_QF && i < C::B_QF + QS                ? 2u        // the copy and the LSE warp
                             : i >= C::B_QE && i < C::B_QE + QS              ? kMmaWarps + kKeyWarps + 0u
                             : i >= C::B_SE && i < C::B_SE + kGroups         ? 4u
                                                                             : 1u);
    *abort_flag = 0;
    ptx::fence_mbar_init();
  }
  if (warp == 0) {
    ptx::tmem_alloc<512>(sbase + C::OFF_MISC);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  Walk walk{begin, end, sp.entry, sp.first};
  Segment s;
  const int n_tiles = (L.d.tokens + L.qt.tokens - 1) / L.qt.tokens;   // query tiles
  bool ok = true;

  if (warp == kWarpK) {
    const int kb = lane % C::KB, sub = lane / C::KB, subs = kKeys / L.box_rows;
    const uint64_t pol = ptx::l2_policy_evict_first();
    uint32_t n = 0;
    while (ok && walk.next(L.c, 1, uc, s, L.status)) {
      for (int t = s.t0; t < s.t1; ++t, ++n) {
        const int st = n % kGroups, key0 = t * kKeys + sub * L.box_rows;
        const bool mine = sub < subs && key0 < s.len;
        const int id = mine ? cache_page(L.c, s.b, s.h, key0 >> L.c.log_page, L.status) : 0;
        if (n >= kGroups && !warp_wait(bar(C::B_KE + st), (n / kGroups - 1) & 1, abort_flag)) {
          ok = false;
          break;
        }
        const int boxes = min(subs, (s.len - t * kKeys + L.box_rows - 1) / L.box_rows) * C::KB;
        if (lane == 0) ptx::mbar_arrive_expect_tx(bar(C::B_KF + st), boxes * L.box_rows * 128);
        __syncwarp();
        if (mine)
          ptx::tma_load_page(sbase + C::OFF_K + st * C::TILE + kb * C::BLOCK + sub * L.box_rows * 128, &L.tm_k,
                             bar(C::B_KF + st), L.k_perm, kb * 64, key0 & (L.c.page - 1), s.h, id, pol);
      }
    }
    if (!ok && lane == 0) record_timeout(abort_flag, L.status);
    const volatile int never = 0;                // no copy in flight at exit
    for (uint32_t i = 0; i < kGroups && i < n; ++i)
      ptx::mbar_wait(bar(C::B_KF + (n - 1 - i) % kGroups), ((n - 1 - i) / kGroups) & 1, &never, kWaitTimeoutNs);
  } else if (warp >= kWarpMma) {
    const int me_w = warp - kWarpMma;            // the units n with n % 2 == me_w
    const int n_cols = (L.qt.rows + 15) & ~15;
    const uint32_t idesc = (1u << 4) | (T::kFormat << 7) | (T::kFormat << 10) | (static_cast<uint32_t>(n_cols >> 3) << 17) |
                           (static_cast<uint32_t>(kKeys >> 4) << 24);
    const uint64_t dk = ptx::sdesc_sw128(sbase + C::OFF_K, 16, 1024), dq = ptx::sdesc_sw128(sbase + C::OFF_Q, 16, 1024);
    uint32_t leader = 0, n = 0, nq = 0, se = 0;  // units, query tiles; parity of the S-empty waits, a bit per group
    int first_leader = -1;
    bool same = true, issued = false;
    while (ok && walk.next(L.c, 1, uc, s, L.status))
      for (int t = s.t0; ok && t < s.t1; t += kGroups) {
        const int count = min(kGroups, s.t1 - t);
        for (int q = 0; ok && q < n_tiles; ++q, ++nq) {
          const int qs = nq % QS;
          ok = warp_wait(bar(C::B_QF + qs), (nq / QS) & 1, abort_flag);
          for (int i = 0; ok && i < count; ++i) {
            const uint32_t st = (n + i) % kGroups;
            if (static_cast<int>(st % kMmaWarps) != me_w) continue;
            // A group's first step finds its buffer free (parity 1 of a fresh barrier passes).
            ok = (q > 0 || warp_wait(bar(C::B_KF + st), ((n + i) / kGroups) & 1, abort_flag)) &&
                 warp_wait(bar(C::B_SE + st), ((se >> st) & 1) ^ 1, abort_flag);
            if (!ok) break;
            se ^= 1u << st;
            ptx::tc_fence_after();
            const bool me = ptx::elect_one(leader);
            if (first_leader < 0) first_leader = static_cast<int>(leader);
            same = same && static_cast<int>(leader) == first_leader;
            if (me && same) {
              const uint64_t kd = dk + static_cast<uint64_t>(st * C::TILE >> 4);
              const uint64_t qd = dq + static_cast<uint64_t>(qs * C::TILE >> 4);
#pragma unroll
              for (int kk = 0; kk < D / 16; ++kk) {
                const uint64_t off = static_cast<uint64_t>(((kk / 4) * C::BLOCK + (kk % 4) * 32) >> 4);
                ptx::mma_ss(tmem + st * 128, kd + off, qd + off, idesc, kk > 0 ? 1u : 0u);
              }
              ptx::mma_commit(bar(C::B_SF + st));
              if (q + 1 == n_tiles) ptx::mma_commit(bar(C::B_KE + st));
            }
            __syncwarp();
            issued = true;
            ok = same;
          }
          // The tile is free once this warp's products with it are done (at once where it had none).
          if (ok) {
            if (ptx::elect_one(leader)) ptx::mma_commit(bar(C::B_QE + qs));
            same = same && (first_leader < 0 || static_cast<int>(leader) == first_leader);
            __syncwarp();
            ok = same;
          }
        }
        n += count;
      }
    if (!ok) {
      if (lane == 0) record_timeout(abort_flag, L.status);
      if (issued && lane == first_leader) {      // every MMA ends before TMEM is released
        const volatile int never = 0;
        ptx::mma_commit(bar(C::B_DRAIN + me_w));
        ptx::mbar_wait(bar(C::B_DRAIN + me_w), 0, &never, kWaitTimeoutNs);
      }
    }
    __syncwarp();
  } else if (warp == kWarpQ) {
    // A tile, and -LSE log2e per row, -inf for a row that does not count. Such a
    // row adds 0 if its logits are finite: its query, which may be anything, is
    // zeroed once it has landed (a test per pair in the sums took 12% of the
    // kernel). A tile's loads are in flight before the tile before it is done, and
    // without branches (serialised, they were the kernel's bound).
    const uint64_t pol = ptx::l2_policy_evict_last();
    int tok_of[4], head_of[4];                   // of this lane's rows, from the tile's first token and head
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = i * 32 + lane;
      tok_of[i] = L.qt.head_inner ? r / L.d.gq : r % L.qt.tokens;
      head_of[i] = L.qt.head_inner ? r % L.d.gq : r / L.qt.tokens;
    }
    struct Rows {
      float lse[4];
      uint8_t use[4];
    };
    int drafted = 0;
    auto load = [&](int q, Rows& x) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int tok = min(q * L.qt.tokens + tok_of[i], L.d.tokens - 1), g = min(head_of[i], L.d.gq - 1);
        const int64_t row = static_cast<int64_t>(s.b) * L.d.tokens + tok;
        x.use[i] = L.use ? __ldg(L.use + row) : 1;
        x.lse[i] = __ldg(L.lse + static_cast<int64_t>(s.h * L.d.gq + g) * L.c.batch * L.d.tokens + row);
      }
    };
    uint32_t n = 0, ql = 0;                      // tiles; parity of the waits for landed ones, a bit per stage
    int open = -1;                               // stage of a tile whose rows are still to be zeroed,
    uint32_t zero = 0;                           // bit i: this lane's i-th row of it
    auto close = [&]() {
      if (open < 0) return;
      ok = ok && warp_wait(bar(C::B_QL + open), (ql >> open) & 1, abort_flag);
      ql ^= 1u << open;
      for (int i = 0; i < 4; ++i)
        if ((zero >> i) & 1)
#pragma unroll
          for (int x = 0; x < C::KB * 8; ++x)
            *reinterpret_cast<uint4*>(smem + C::OFF_Q + open * C::TILE + (x / 8) * C::BLOCK + (i * 32 + lane) * 128 + (x % 8) * 16) =
                make_uint4(0, 0, 0, 0);
      ptx::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(bar(C::B_QF + open));
      open = -1;
    };
    while (ok && walk.next(L.c, 1, uc, s, L.status)) {
      drafted = drafted_tokens(L.d, s.b);
      Rows now, next;
      load(0, next);
      for (int t = s.t0; ok && t < s.t1; t += kGroups)
        for (int q = 0; ok && q < n_tiles; ++q, ++n) {
          const int st = n % QS;
          now = next;
          if (n_tiles > 1) load(q + 1 < n_tiles ? q + 1 : 0, next);
          float v[4];
          uint32_t drop = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int tok = q * L.qt.tokens + tok_of[i];
            const bool row = i * 32 + lane < L.qt.rows;
            const bool in = row && tok < drafted && now.use[i] != 0 && now.lse[i] != -INFINITY;
            v[i] = in ? -kLog2e * now.lse[i] : -INFINITY;
            drop |= static_cast<uint32_t>(row && !in) << i;
          }
          const bool part = __any_sync(0xffffffffu, drop != 0);
          if (n >= QS) {
            if (!__all_sync(0xffffffffu, ptx::mbar_test(bar(C::B_QE + st), (n / QS - 1) & 1))) close();
            ok = ok && warp_wait(bar(C::B_QE + st), (n / QS - 1) & 1, abort_flag);
            if (!ok) break;
          }
          if (lane == 0) {
            const uint32_t landed = bar((part ? C::B_QL : C::B_QF) + st);
            ptx::mbar_arrive_expect_tx(landed, C::KB * L.qt.rows * 128);
            for (int kb = 0; kb < C::KB; ++kb)
              ptx::tma_load_page(sbase + C::OFF_Q + st * C::TILE + kb * C::BLOCK, &L.tm_q, landed, L.q_perm, kb * 64,
                                 q * L.qt.tokens, s.h * L.d.gq, s.b, pol);
          }
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 4; ++i) lse_s[st * 128 + i * 32 + lane] = v[i];
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(bar(C::B_QF + st));
          close();
          if (part) {
            open = st;
            zero = drop;
          }
        }
    }
    close();
    if (!ok && lane == 0) record_timeout(abort_flag, L.status);
    // No copy in flight at exit: after a failure the last tiles' phases may never
    // complete (their other arrival is missing), and these waits end by their limit.
    const volatile int never = 0;
    for (uint32_t i = 0; i < QS && i < n; ++i)
      ptx::mbar_wait(bar(C::B_QF + (n - 1 - i) % QS), ((n - 1 - i) / QS) & 1, &never, kWaitTimeoutNs);
  } else {
    const int grp = warp >> 2, key = threadIdx.x & 127;
    const uint32_t tS = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + grp * 128;
    const uint64_t scale2 = ptx::f2(L.d.scale_log2, L.d.scale_log2);
    uint32_t n = 0, nq = 0, step = 0;
    while (walk.next(L.c, 1, uc, s, L.status))
      for (int t = s.t0; t < s.t1; t += kGroups) {
        const int count = min(kGroups, s.t1 - t), mine = (grp - n) & (kGroups - 1);
        n += count;
        const bool active = mine < count;
        const int64_t pos = static_cast<int64_t>(t + mine) * kKeys + key;
        const bool live = active && pos < s.len && pos < L.acc_len;
        if (active && pos < s.len && pos >= L.acc_len) record_bounds(L.status);
        float* dst = L.acc + (static_cast<int64_t>(s.b) * L.c.hkv + s.h) * L.acc_len + pos;
        const float old = live && L.accumulate ? *dst : 0.f;
        uint64_t a2[4] = {0, 0, 0, 0};
        for (int q = 0; q < n_tiles; ++q, ++nq) {
          const int qs = nq % QS;
          ok = ok && warp_wait(bar(C::B_QF + qs), (nq / QS) & 1, abort_flag);
          if (active) {
            ok = ok && warp_wait(bar(C::B_SF + grp), step & 1, abort_flag);
            ++step;
            if (ok) {
              ptx::tc_fence_after();
              const float* lrow = lse_s + qs * 128;
              const int valid = L.qt.head_inner ? min(L.qt.rows, (L.d.tokens - q * L.qt.tokens) * L.d.gq) : L.qt.rows;
              auto add4 = [&](const uint32_t* r, const float4& nl, int e) {
                float x0, x1, x2, x3;
                ptx::unf2(ptx::fma2(ptx::f2(__uint_as_float(r[0]), __uint_as_float(r[1])), scale2, ptx::f2(nl.x, nl.y)), x0, x1);
                ptx::unf2(ptx::fma2(ptx::f2(__uint_as_float(r[2]), __uint_as_float(r[3])), scale2, ptx::f2(nl.z, nl.w)), x2, x3);
                a2[(2 * e) & 3] = ptx::add2(a2[(2 * e) & 3], ptx::f2(ptx::ex2(x0), ptx::ex2(x1)));
                a2[(2 * e + 1) & 3] = ptx::add2(a2[(2 * e + 1) & 3], ptx::f2(ptx::ex2(x2), ptx::ex2(x3)));
              };
              int c0 = 0;
#pragma unroll 1
              for (; c0 + 32 <= valid; c0 += 32) {
                float4 l4[8];                    // read before the TMEM wait, which covers their latency
                uint32_t r[32];
                ptx::tmem_ld32(tS + c0, r);
#pragma unroll
                for (int e = 0; e < 8; ++e) l4[e] = reinterpret_cast<const float4*>(lrow + c0)[e];
                ptx::tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 8; ++e) add4(r + 4 * e, l4[e], e);
              }
              // The last columns by 16; past the tile's rows they are whatever its stage held.
#pragma unroll 1
              for (; c0 < valid; c0 += 16) {
                float4 l4[4];
                uint32_t r[16];
                ptx::tmem_ld16(tS + c0, r);
#pragma unroll
                for (int e = 0; e < 4; ++e) l4[e] = reinterpret_cast<const float4*>(lrow + c0)[e];
                ptx::tmem_wait_ld();
                if (c0 + 16 > valid) {
#pragma unroll
                  for (int e = 1; e < 16; ++e)
                    if (c0 + e >= valid) r[e] = 0u;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) add4(r + 4 * e, l4[e], e);
              }
              ptx::tc_fence_before();
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(bar(C::B_SE + grp));
          }
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(bar(C::B_QE + qs));
        }
        float s0, s1, s2, s3;
        ptx::unf2(ptx::add2(a2[0], a2[1]), s0, s1);
        ptx::unf2(ptx::add2(a2[2], a2[3]), s2, s3);
        float sum = (s0 + s1) + (s2 + s3);
        if (live && isnan(sum)) sum = counted_sum<T, D>(L, s.b, s.h, static_cast<int>(pos));
        if (ok && live) *dst = old + sum;
      }
    if (!ok && lane == 0) record_timeout(abort_flag, L.status);
  }
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc<512>(tmem);
  }
}

// Queries that a TMA map cannot describe (a dimension repeated by a stride of 0),
// or none at all: one thread per key, every row read again (128 tokens of 7 heads over
// 65,536 keys: 15.4 ms).
constexpr int kPlainThreads = 128;

template <class T, int D>
__global__ void __launch_bounds__(kPlainThreads) cache_evidence_plain_kernel(const __grid_constant__ CacheEvidenceLaunch L) {
  const int h = blockIdx.y, b = blockIdx.z, key = blockIdx.x * kPlainThreads + threadIdx.x;
  int len = cache_len(L.c, b, h, L.status);
  if (len > L.acc_len) {
    record_bounds(L.status);
    len = static_cast<int>(L.acc_len);
  }
  if (key >= len) return;
  const float sum = counted_sum<T, D>(L, b, h, key);
  float* dst = L.acc + (static_cast<int64_t>(b) * L.c.hkv + h) * L.acc_len + key;
  *dst = L.accumulate ? *dst + sum : sum;
}

template <class T, int D>
cudaError_t launch_d(const CacheEvidenceLaunch& L, cudaStream_t stream) {
  if (L.has_q_map) {
    using C = EvCfg<D>;
    auto kern = cache_evidence_kernel<T, D>;
    static PerDeviceAttr once;
    const cudaError_t e = raise_smem_limit(once, reinterpret_cast<const void*>(kern), C::SMEM);
    if (e != cudaSuccess) return e;
    return launch_after(kern, dim3(L.n_ctas), kThreads, C::SMEM, stream, L);
  }
  const int64_t room = static_cast<int64_t>(L.c.max_pages) * L.c.page;
  const dim3 grid(static_cast<unsigned>((room + kPlainThreads - 1) / kPlainThreads), L.c.hkv, L.c.batch);
  cache_evidence_plain_kernel<T, D><<<grid, kPlainThreads, 0, stream>>>(L);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_cache_evidence(const CacheEvidenceLaunch& L, cudaStream_t stream) {
  if (L.c.dtype == 0) return L.c.head_dim == 128 ? launch_d<BF16, 128>(L, stream) : launch_d<BF16, 64>(L, stream);
  return L.c.head_dim == 128 ? launch_d<FP16, 128>(L, stream) : launch_d<FP16, 64>(L, stream);
}

}  // namespace evisel
