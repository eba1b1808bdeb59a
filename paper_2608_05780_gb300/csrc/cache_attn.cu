// Attention of drafted tokens over a paged cache: partial results of ranges of
// cached keys, and their join with the drafted tokens' own attention.
//
//   s_rm = scale q_r . k_m,  O_r = sum_m exp(s_rm - LSE_r) v_m
//
// over a (sequence, KV head)'s rows r = (token, head of the group).
#include <algorithm>
#include <cstdint>
#include <cuda_runtime.h>

#include "cache_attn.cuh"

namespace evisel {
namespace {

constexpr float kLn2 = 0.69314718055994531f;
constexpr int kKeys = 64;                        // keys of a unit
constexpr int kKeyWarps = 4;                     // warps over a unit's keys, 16 each
constexpr int kStages = 3;

// ---------------------------------------------------------------- few rows
// Up to 16 * MG rows of a (sequence, KV head) at a time. Each of four warps takes
// 16 of a unit's 64 keys against all rows with a running max, row sum and O of
// its own (mma.sync, fp32 accumulators in registers, two CTAs per SM); they are
// joined when the CTA leaves the problem. A producer warp streams the pages by TMA.
// P is rounded to 16 bits for its product with V, since that is what the tensor
// cores multiply by the cache's type (O off by 2.3e-3 against 1.7e-3 in bf16,
// 2.1e-4 against 2.0e-4 in fp16); its sum is not.
// The stream is the bound: one token of 32 sequences of up to 16,512 (581 MB) takes 91 us,
// 94% of a plain copy's rate, with the tensor pipe 18% busy. Little work is latency:
// one token over 4,160 tokens about 4 us of launch, lengths, table and first loads.
template <int D, int MG>
struct FewCfg {
  static constexpr int KB = D / 64;                          // 128-byte column blocks
  static constexpr int BLOCK = kKeys * 128;                  // one column block of a unit
  static constexpr int TILE = KB * BLOCK;
  static constexpr int OFF_K = 0;
  static constexpr int OFF_V = kStages * TILE;
  // MG = 2: a segment's 32 queries, swizzled like K; then, at its end, 16 rows x D fp32.
  static constexpr int OFF_Q = 2 * kStages * TILE, OFF_JOIN = OFF_Q;
  static constexpr int OFF_ML = OFF_JOIN + 16 * D * 4;       // per key warp: 16 MG x (max, sum)
  static_assert(16 * MG * D * 2 <= 16 * D * 4, "the queries fit where the join goes");
  static constexpr int OFF_BAR = OFF_ML + MG * kKeyWarps * 16 * 8;
  static constexpr int B_FULL = 0, B_EMPTY = kStages;
  static constexpr int OFF_MISC = OFF_BAR + 2 * kStages * 8; // abort flag, split scratch
  static constexpr int SMEM = OFF_MISC + 8 + 40 * 4 + 1024;
  static constexpr int THREADS = 32 * (kKeyWarps + 1);
  static_assert(2 * (SMEM + 1024) <= 233472, "two CTAs per SM");
};

template <class T, int D, int MG>
__global__ void __launch_bounds__(32 * (kKeyWarps + 1), 2) cache_attn_few_kernel(const __grid_constant__ CacheAttnLaunch L) {
  using C = FewCfg<D, MG>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t sbase = ptx::smem_addr(smem);
  auto bar = [&](int i) { return sbase + C::OFF_BAR + 8u * i; };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::OFF_MISC);
  int* scratch = reinterpret_cast<int*>(smem + C::OFF_MISC + 8);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      ptx::mbar_init(bar(C::B_FULL + i), 1);
      ptx::mbar_init(bar(C::B_EMPTY + i), kKeyWarps);
    }
    *abort_flag = 0;
    ptx::fence_mbar_init();
  }
  if (threadIdx.x == 0 && L.c.max_pages > 0) {   // (without any page there is no map)
    ptx::tma_prefetch_desc(&L.tm_k);
    ptx::tma_prefetch_desc(&L.tm_v);
  }
  ptx::grid_wait();
  ptx::grid_launch_next();
  const UnitCount uc(L.c, kKeys, L.lead, L.row_tiles, L.status);
  int ctas = 1, end = 0;
  const Split sp = split_find_unit(uc, scratch, [&](int total) {
    ctas = split_ctas(total, L.n_ctas, L.min_units, L.c.batch * L.c.hkv * L.row_tiles);
    const int i = blockIdx.x;
    end = i < ctas ? split_begin(i + 1, total, ctas) : 0;
    return i < ctas ? split_begin(i, total, ctas) : total;
  });
  const int begin = static_cast<int>(blockIdx.x) < ctas ? split_begin(blockIdx.x, sp.total, ctas) : sp.total;
  if (begin >= end) return;                      // (the whole block: nothing was started)
  Walk walk{begin, end, sp.entry, sp.first};
  Segment s;
  uint32_t n = 0;                                // units so far
  bool ok = true;

  if (warp == kKeyWarps) {
    // Producer: lane i sends one box of K or V.
    const int subs = kKeys / L.box_rows, n_loads = subs * C::KB * 2;
    const int sub = lane / (2 * C::KB), kb = (lane >> 1) % C::KB, is_v = lane & 1;
    const CUtensorMap* map = is_v ? &L.tm_v : &L.tm_k;
    const int perm = is_v ? L.v_perm : L.k_perm;
    const uint64_t pol = ptx::l2_policy_evict_first();
    while (ok && walk.next(L.c, L.row_tiles, uc, s, L.status)) {
      for (int t = s.t0; t < s.t1; ++t, ++n) {
        const int st = n % kStages, key0 = t * kKeys + sub * L.box_rows;
        const bool mine = lane < n_loads && key0 < s.len;
        const int id = mine ? cache_page(L.c, s.b, s.h, key0 >> L.c.log_page, L.status) : 0;
        if (n >= kStages && !warp_wait(bar(C::B_EMPTY + st), (n / kStages - 1) & 1, abort_flag)) {
          ok = false;
          break;
        }
        const int boxes = min(subs, (s.len - t * kKeys + L.box_rows - 1) / L.box_rows) * C::KB * 2;
        if (lane == 0) ptx::mbar_arrive_expect_tx(bar(C::B_FULL + st), boxes * L.box_rows * 128);
        __syncwarp();
        if (mine)
          ptx::tma_load_page(sbase + (is_v ? C::OFF_V : C::OFF_K) + st * C::TILE + kb * C::BLOCK + sub * L.box_rows * 128,
                             map, bar(C::B_FULL + st), perm, kb * 64, key0 & (L.c.page - 1), s.h, id, pol);
      }
    }
    if (!ok && lane == 0) record_timeout(abort_flag, L.status);
    // no copy in flight at exit
    const volatile int never = 0;
    for (uint32_t i = 0; i < kStages && i < n; ++i)
      ptx::mbar_wait(bar(C::B_FULL + (n - 1 - i) % kStages), ((n - 1 - i) / kStages) & 1, &never, kWaitTimeoutNs);
    return;
  }

  const int kw = warp;
  const int r8 = lane & 7, mi = lane >> 3;
  // ldmatrix addresses within a tile: this lane's row, and its 16-byte chunk at even k-steps (^ swizzle).
  const int k_row = kw * 16 + (mi >> 1) * 8 + r8, k_chunk = mi & 1;
  const int v_row = kw * 16 + (mi & 1) * 8 + r8, v_chunk = mi >> 1;
  const int q_row = (mi & 1) * 8 + r8, q_chunk = mi >> 1;
  const int fr = lane >> 2, fc = (lane & 3) * 2;  // fragment row (and row + 8) and first column
  constexpr int QBLOCK = 16 * MG * 128;
  float4* join = reinterpret_cast<float4*>(smem + C::OFF_JOIN);
  float2* ml = reinterpret_cast<float2*>(smem + C::OFF_ML);

  while (walk.next(L.c, L.row_tiles, uc, s, L.status)) {
    // The rows' queries (zeros past the last row): 16 rows as fragments in
    // registers, 32 in shared memory, where their fragments are read per unit.
    [[maybe_unused]] uint32_t qf[MG == 1 ? D / 16 : 1][4];
    const uint16_t* qb = static_cast<const uint16_t*>(L.d.q) + s.b * L.d.qs[0] + s.h * L.d.gq * L.d.qs[2];
    if constexpr (MG == 1) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int r = s.rt * L.tile_rows + fr + half * 8;
        const bool in = r < L.rows;
        const int t = in ? r / L.d.gq : 0, g = in ? r % L.d.gq : 0;
        const uint32_t* q = reinterpret_cast<const uint32_t*>(qb + t * L.d.qs[1] + g * L.d.qs[2] + fc);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          qf[ks][half] = in ? __ldg(q + ks * 8) : 0u;
          qf[ks][half + 2] = in ? __ldg(q + ks * 8 + 4) : 0u;
        }
      }
    } else {
      ptx::bar_sync(1, 32 * kKeyWarps);          // the last segment's queries have been read
      for (int i = threadIdx.x; i < 16 * MG * D / 8; i += 32 * kKeyWarps) {
        const int row = i / (D / 8), ch = i % (D / 8), r = s.rt * L.tile_rows + row;
        const bool in = r < L.rows;
        const int t = in ? r / L.d.gq : 0, g = in ? r % L.d.gq : 0;
        const uint4 x = in ? __ldg(reinterpret_cast<const uint4*>(qb + t * L.d.qs[1] + g * L.d.qs[2]) + ch) : make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(smem + C::OFF_Q + (ch / 8) * QBLOCK + row * 128 + ((ch & 7) ^ (row & 7)) * 16) = x;
      }
      ptx::bar_sync(1, 32 * kKeyWarps);
    }
    float o[MG][D / 8][4];
    float m[MG][2], l[MG][2];
#pragma unroll
    for (int g = 0; g < MG; ++g) {
#pragma unroll
      for (int j = 0; j < D / 8; ++j) o[g][j][0] = o[g][j][1] = o[g][j][2] = o[g][j][3] = 0.f;
      m[g][0] = m[g][1] = -INFINITY;
      l[g][0] = l[g][1] = 0.f;
    }

    for (int t = s.t0; t < s.t1; ++t, ++n) {
      const int st = n % kStages;
      ok = ok && warp_wait(bar(C::B_FULL + st), (n / kStages) & 1, abort_flag);
      const int left = s.len - t * kKeys - kw * 16;   // keys of this warp that exist
      if (ok && left > 0) {
        const uint32_t kt = sbase + C::OFF_K + st * C::TILE, vt = sbase + C::OFF_V + st * C::TILE;
        float sc[MG][2][4] = {};
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          uint32_t kf[4];
          const int ch = (ks % 4) * 2 + k_chunk;
          ptx::ldmatrix4(kf, kt + (ks / 4) * C::BLOCK + k_row * 128 + ((ch ^ r8) << 4));
#pragma unroll
          for (int g = 0; g < MG; ++g) {
            uint32_t qr[4];
            if constexpr (MG == 1) {
#pragma unroll
              for (int e = 0; e < 4; ++e) qr[e] = qf[ks][e];
            } else {
              const int qch = (ks % 4) * 2 + q_chunk;
              ptx::ldmatrix4(qr, sbase + C::OFF_Q + (ks / 4) * QBLOCK + (g * 16 + q_row) * 128 + ((qch ^ r8) << 4));
            }
            ptx::mma16816<T>(sc[g][0], qr, kf[0], kf[1]);
            ptx::mma16816<T>(sc[g][1], qr, kf[2], kf[3]);
          }
        }
        if (left < 16) {
          // Past the sequence's end: the keys are masked, and their values, which
          // may be anything, are zeroed (each warp reads its own 16 rows only).
#pragma unroll
          for (int g = 0; g < MG; ++g)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (j * 8 + fc + (e & 1) >= left) sc[g][j][e] = -INFINITY;
          for (int i = lane; i < (16 - left) * C::KB * 8; i += 32) {
            const int row = kw * 16 + left + i / (C::KB * 8), x = i % (C::KB * 8);
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(vt + (x / 8) * C::BLOCK + row * 128 + (x % 8) * 16),
                         "r"(0)
                         : "memory");
          }
          ptx::fence_proxy_async_smem();
          __syncwarp();
        }
        // Running max (log2 units, less the headroom), moved only when it grows by more than 2^8.
        float tm[MG][2];
        bool grows = false;
#pragma unroll
        for (int g = 0; g < MG; ++g)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            float x = fmaxf(fmaxf(sc[g][0][2 * half], sc[g][0][2 * half + 1]), fmaxf(sc[g][1][2 * half], sc[g][1][2 * half + 1]));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
            tm[g][half] = fmaf(x, L.d.scale_log2, -T::kHeadroom);
            grows = grows || tm[g][half] > m[g][half] + kRescaleThreshold;
          }
        if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
          for (int g = 0; g < MG; ++g)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const bool need = tm[g][half] > m[g][half] + kRescaleThreshold;
              const float alpha = need ? ptx::ex2(m[g][half] - tm[g][half]) : 1.f;
              if (need) m[g][half] = tm[g][half];
              l[g][half] *= alpha;
#pragma unroll
              for (int j = 0; j < D / 8; ++j) {
                o[g][j][2 * half] *= alpha;
                o[g][j][2 * half + 1] *= alpha;
              }
            }
        }
        uint32_t pa[MG][4];
#pragma unroll
        for (int g = 0; g < MG; ++g) {
          const float ms[2] = {m[g][0] == -INFINITY ? 0.f : m[g][0], m[g][1] == -INFINITY ? 0.f : m[g][1]};
          float p[2][4];
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              p[j][e] = ptx::ex2(fmaf(sc[g][j][e], L.d.scale_log2, -ms[e >> 1]));
              l[g][e >> 1] += p[j][e];
            }
          pa[g][0] = T::pack(p[0][0], p[0][1]);
          pa[g][1] = T::pack(p[0][2], p[0][3]);
          pa[g][2] = T::pack(p[1][0], p[1][1]);
          pa[g][3] = T::pack(p[1][2], p[1][3]);
        }
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
          uint32_t vf[4];
          const int ch = (j % 4) * 2 + v_chunk;
          ptx::ldmatrix4_t(vf, vt + (j / 4) * C::BLOCK + v_row * 128 + ((ch ^ r8) << 4));
#pragma unroll
          for (int g = 0; g < MG; ++g) {
            ptx::mma16816<T>(o[g][2 * j], pa[g], vf[0], vf[1]);
            ptx::mma16816<T>(o[g][2 * j + 1], pa[g], vf[2], vf[3]);
          }
        }
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(bar(C::B_EMPTY + st));
    }

    // Join of the four key warps (every warp passes every barrier, also after a
    // failure), and the partial of this segment.
#pragma unroll
    for (int g = 0; g < MG; ++g)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        l[g][half] += __shfl_xor_sync(0xffffffffu, l[g][half], 1);
        l[g][half] += __shfl_xor_sync(0xffffffffu, l[g][half], 2);
        if ((lane & 3) == 0) ml[(kw * MG + g) * 16 + fr + 8 * half] = make_float2(m[g][half], l[g][half]);
      }
    ptx::bar_sync(1, 32 * kKeyWarps);
    const int64_t part0 = (static_cast<int64_t>(blockIdx.x) + s.problem) * L.tile_rows;
#pragma unroll
    for (int g = 0; g < MG; ++g) {
      float top[2], sum[2], f[2];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        top[half] = -INFINITY;
        sum[half] = 0.f;
#pragma unroll
        for (int w = 0; w < kKeyWarps; ++w) top[half] = fmaxf(top[half], ml[(w * MG + g) * 16 + fr + 8 * half].x);
        const float ref = top[half] == -INFINITY ? 0.f : top[half];
#pragma unroll
        for (int w = 0; w < kKeyWarps; ++w) {
          const float2 x = ml[(w * MG + g) * 16 + fr + 8 * half];
          sum[half] += x.y * ptx::ex2(x.x - ref);
        }
        f[half] = ptx::ex2(m[g][half] - ref);
      }
#pragma unroll
      for (int j = 0; j < D / 8; ++j) {
        o[g][j][0] *= f[0], o[g][j][1] *= f[0], o[g][j][2] *= f[1], o[g][j][3] *= f[1];
      }
#pragma unroll
      for (int w = kKeyWarps - 1; w >= 0; --w) {
        if (kw == w) {
#pragma unroll
          for (int j = 0; j < D / 8; ++j) {
            if (w < kKeyWarps - 1) {
              const float4 x = join[j * 32 + lane];
              o[g][j][0] += x.x, o[g][j][1] += x.y, o[g][j][2] += x.z, o[g][j][3] += x.w;
            }
            if (w > 0) join[j * 32 + lane] = make_float4(o[g][j][0], o[g][j][1], o[g][j][2], o[g][j][3]);
          }
        }
        if (w > 0 || g + 1 < MG) ptx::bar_sync(1, 32 * kKeyWarps);
      }
      if (kw == 0 && ok) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int64_t row = part0 + g * 16 + fr + 8 * half;
          float* dst = L.part_o + row * D + fc;
#pragma unroll
          for (int j = 0; j < D / 8; ++j)
            *reinterpret_cast<float2*>(dst + j * 8) = make_float2(o[g][j][2 * half], o[g][j][2 * half + 1]);
          if ((lane & 3) == 0) L.part_ml[row] = make_float2(top[half], sum[half]);
        }
      }
    }
  }
  if (!ok && lane == 0) record_timeout(abort_flag, L.status);
}

// ---------------------------------------------------------------- join
// One row of a (sequence, KV head): its partials, and its own attention over the
// drafted tokens that its bits allow (only those are read, so that values of
// the others never enter). A row is shared by `wpr` warps, each with a running
// max of its own. Dependent loads are the bound: 10 us by itself for 896 rows of 3 partials,
// of which the drafted half runs before the kernel that it follows has ended.
constexpr int kJoinWarps = 8;

// LSE of a row sum l relative to 2^m.
template <class T>
__device__ __forceinline__ float row_lse(float m, float l) {
  constexpr float kDown = T::kHeadroom > 0.f ? 0x1p-7f : 1.f;    // (lg2 is the more exact the nearer to 1)
  static_assert(T::kHeadroom == 0.f || T::kHeadroom == 7.f, "kDown");
  return l != 0.f ? ((m + T::kHeadroom) + __log2f(l * kDown)) * kLn2 : -INFINITY;
}

template <class T, int D>
__global__ void __launch_bounds__(32 * kJoinWarps, 4) cache_join_kernel(const __grid_constant__ CacheAttnLaunch L, int wpr) {
  constexpr int E = D / 32;                      // elements of a row per lane
  __shared__ int scratch[40];
  __shared__ float join_o[kJoinWarps][D];
  __shared__ float2 join_ml[kJoinWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int bh = blockIdx.y, b = bh / L.c.hkv, h = bh % L.c.hkv;
  // Everything but the partials was there before the kernel that this one follows began.
  const UnitCount uc(L.c, L.key_tile, L.lead, L.row_tiles, L.status);
  const Split sp = split_find_entry(uc, scratch, uc.per_head ? bh : b);
  const int tiles = uc.tiles(sp.entry);
  const int first = sp.first + (uc.per_head ? 0 : h * L.row_tiles * uc.units(tiles));
  const int ctas = split_ctas(sp.total, L.n_ctas, L.min_units, L.c.batch * L.c.hkv * L.row_tiles);

  const int r = blockIdx.x * (kJoinWarps / wpr) + warp / wpr, wi = warp % wpr;
  const bool in = r < L.rows;
  const int t = in ? r / L.d.gq : 0, g = in ? r % L.d.gq : 0, head = h * L.d.gq + g;
  const int drafted = drafted_tokens(L.d, b);
  const bool live = in && t < drafted;
  float m = -INFINITY, l = 0.f, acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  auto move_max = [&](float x) {                 // the running max is at least x from here on
    if (x > m) {
      const float a = ptx::ex2(m - x);
      l *= a;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] *= a;
      m = x;
    }
  };

  // The drafted tokens first: they need nothing of the kernel before.
  if (live && L.d.k_new) {
    auto load = [&](const void* base, const int64_t (&st)[3], int tok, int hd, float (&x)[E]) {
      const uint16_t* p = static_cast<const uint16_t*>(base) + b * st[0] + tok * st[1] + hd * st[2] + lane * E;
      if constexpr (E == 4) {
        const uint2 y = __ldg(reinterpret_cast<const uint2*>(p));
        x[0] = T::lo(y.x), x[1] = T::hi(y.x), x[2] = T::lo(y.y), x[3] = T::hi(y.y);
      } else {
        const uint32_t y = __ldg(reinterpret_cast<const uint32_t*>(p));
        x[0] = T::lo(y), x[1] = T::hi(y);
      }
    };
    float q[E];
    load(L.d.q, L.d.qs, t, head, q);
    const int words = (drafted + 31) / 32;
    for (int w = 0; w < words; ++w) {
      uint32_t bits = L.d.tree ? static_cast<uint32_t>(__ldg(L.d.tree + b * L.d.trs[0] + t * L.d.trs[1] + w))
                      : t - 32 * w >= 31 ? 0xffffffffu
                      : t < 32 * w       ? 0u
                                         : (2u << (t - 32 * w)) - 1u;
      if (drafted - 32 * w < 32) bits &= (1u << (drafted - 32 * w)) - 1u;
      // This warp's share of the bits: its eighth, quarter or half of the word's places.
      const uint32_t every = wpr == 8 ? 0x01010101u : wpr == 4 ? 0x11111111u : wpr == 2 ? 0x55555555u : 0xffffffffu;
      bits &= every << wi;
      // Four keys at a time: their loads together, their four sums over the lanes in one exchange.
      while (bits) {
        int tok[4];
        bool on[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          on[i] = bits != 0;
          tok[i] = 32 * w + (on[i] ? __ffs(bits) - 1 : 0);
          bits &= bits - 1;
        }
        float k[4][E], v[4][E], x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (!on[i]) tok[i] = tok[0];
          load(L.d.k_new, L.d.kns, tok[i], h, k[i]);
          load(L.d.v_new, L.d.vns, tok[i], h, v[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) x[i] = fmaf(q[e], k[i][e], x[i]);
        }
        const bool hi = lane & 16, mid = lane & 8;
        const float y0 = (hi ? x[2] : x[0]) + __shfl_xor_sync(0xffffffffu, hi ? x[0] : x[2], 16);
        const float y1 = (hi ? x[3] : x[1]) + __shfl_xor_sync(0xffffffffu, hi ? x[1] : x[3], 16);
        float z = (mid ? y1 : y0) + __shfl_xor_sync(0xffffffffu, mid ? y0 : y1, 8);
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
        z *= L.d.scale_log2;                     // lanes 8 i .. 8 i + 7: key i
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = __shfl_sync(0xffffffffu, z, 8 * i);
          if (on[i]) top = fmaxf(top, x[i]);
        }
        move_max(top);
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (on[i]) {
            const float p = ptx::ex2(x[i] - ref);
            l += p;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = fmaf(p, v[i][e], acc[e]);
          }
      }
    }
  }

  ptx::grid_wait();
  ptx::grid_launch_next();
  if (live && tiles > 0) {
    const int slot = r / L.slot_rows, rt = slot / L.slots;
    const int in_slot = L.wide && !L.qt.head_inner ? g * L.qt.tokens + t % L.qt.tokens : r % L.slot_rows;
    const int row = (slot % L.slots) * (L.tile_rows / L.slots) + in_slot;
    const int u0 = first + rt * uc.units(tiles) + uc.lead, i0 = split_owner(u0, sp.total, ctas), i1 = split_owner(u0 + tiles - 1, sp.total, ctas);
    const int problem = bh * L.row_tiles + rt;
    const int n = (i1 - i0 + 1 - wi + wpr - 1) / wpr;            // partials of this warp
    const int64_t step = static_cast<int64_t>(wpr) * L.tile_rows;
    const int64_t row0 = static_cast<int64_t>(i0 + problem + wi) * L.tile_rows + row;
    // Eight partials at a time, all loads at once.
    for (int base = 0; base < n; base += 8) {
      float y[8][E];
      const float2 x = lane < 8 && base + lane < n ? L.part_ml[row0 + (base + lane) * step] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float* src = L.part_o + (row0 + (base + k) * step) * D + lane * E;
        if (base + k < n) {
          if constexpr (E == 4) {
            const float4 z = *reinterpret_cast<const float4*>(src);
            y[k][0] = z.x, y[k][1] = z.y, y[k][2] = z.z, y[k][3] = z.w;
          } else {
            const float2 z = *reinterpret_cast<const float2*>(src);
            y[k][0] = z.x, y[k][1] = z.y;
          }
        }
      }
      float top = x.x;
#pragma unroll
      for (int o = 4; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      move_max(__shfl_sync(0xffffffffu, top, 0));
      const float w = ptx::ex2(x.x - (m == -INFINITY ? 0.f : m)), lw = x.y * w;
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (base + k < n) {
          const float wk = __shfl_sync(0xffffffffu, w, k);
          l += __shfl_sync(0xffffffffu, lw, k);
#pragma unroll
          for (int e = 0; e < E; ++e) acc[e] = fmaf(wk, y[k][e], acc[e]);
        }
    }
  }
  if (wpr > 1) {
#pragma unroll
    for (int e = 0; e < E; ++e) join_o[warp][lane * E + e] = acc[e];
    if (lane == 0) join_ml[warp] = make_float2(m, l);
    __syncthreads();
    if (wi == 0)
      for (int w = 1; w < wpr; ++w) {
        const float2 x = join_ml[warp + w];
        move_max(x.x);
        const float f = ptx::ex2(x.x - (m == -INFINITY ? 0.f : m));
        l += x.y * f;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += f * join_o[warp + w][lane * E + e];
      }
  }
  if (!in || wi != 0) return;
  const float inv = l != 0.f ? 1.f / l : 0.f;    // (a NaN sum stays one)
  uint16_t* dst = static_cast<uint16_t*>(L.o) + ((static_cast<int64_t>(b) * L.d.tokens + t) * L.d.hq + head) * D + lane * E;
  if constexpr (E == 4)
    *reinterpret_cast<uint2*>(dst) = make_uint2(T::pack(acc[0] * inv, acc[1] * inv), T::pack(acc[2] * inv, acc[3] * inv));
  else
    *reinterpret_cast<uint32_t*>(dst) = T::pack(acc[0] * inv, acc[1] * inv);
  if (lane == 0)
    L.lse[(static_cast<int64_t>(head) * L.c.batch + b) * L.d.tokens + t] = row_lse<T>(m, l);
}

// Many rows: 16 of them a warp as one side of mma.sync products, the drafted keys
// staged in shared memory for the block's rows. Masked keys' products never count;
// their values meet weights of 0, so a block whose drafted values are not all
// finite takes its P V value by value, over the allowed ones only. P is rounded to 16
// bits for the product, its sum is not. `wpr` warps share 16 rows.
// 24 drafted tokens of 32 sequences (21,504 rows, 38 MB of partials, mostly in L2, and
// results): 18.4 us by itself, 45 row by row; the loads of the partials are the bound.
constexpr int kTileWarps = 4, kChunk = 64;

template <class T>
__device__ __forceinline__ bool all_finite(const uint4& x) {
  constexpr uint32_t kExp = T::kFormat == 1 ? 0x7f80u : 0x7c00u;
  bool ok = true;
#pragma unroll
  for (uint32_t w : {x.x, x.y, x.z, x.w}) ok = ok && (w & kExp) != kExp && ((w >> 16) & kExp) != kExp;
  return ok;
}

template <class T, int D>
__global__ void __launch_bounds__(32 * kTileWarps, 3) cache_join_tile_kernel(const __grid_constant__ CacheAttnLaunch L, int wpr) {
  constexpr int BLOCK = kChunk * 128, KB = D / 64;           // a 64-column block of a chunk
  constexpr float kHeadroom = T::kHeadroom > 0.f ? T::kHeadroom + kRescaleThreshold : 0.f;  // (this maximum is never stale)
  __shared__ alignas(128) uint8_t tile[2 * KB * BLOCK];      // drafted keys and values, swizzled; then the warps' O
  __shared__ float2 join_ml[kTileWarps][16];
  __shared__ int scratch[40];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wi = warp % wpr, group = warp / wpr;
  const int bh = blockIdx.y, b = bh / L.c.hkv, h = bh % L.c.hkv;
  // Everything but the partials was there before the kernel that this one follows began.
  const UnitCount uc(L.c, L.key_tile, L.lead, L.row_tiles, L.status);
  const Split sp = split_find_entry(uc, scratch, uc.per_head ? bh : b);
  const int tiles = uc.tiles(sp.entry);
  const int first = sp.first + (uc.per_head ? 0 : h * L.row_tiles * uc.units(tiles));
  const int ctas = split_ctas(sp.total, L.n_ctas, L.min_units, L.c.batch * L.c.hkv * L.row_tiles);
  const int drafted = drafted_tokens(L.d, b);

  const int fr = lane >> 2, fc = (lane & 3) * 2, mi = lane >> 3, r8 = lane & 7;
  const int block0 = blockIdx.x * (kTileWarps / wpr) * 16;
  int r[2], t[2];
  bool in[2], live[2];
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    r[half] = block0 + group * 16 + fr + 8 * half;
    in[half] = r[half] < L.rows;
    t[half] = in[half] ? r[half] / L.d.gq : 0;
    live[half] = in[half] && t[half] < drafted;
  }
  float o[D / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int j = 0; j < D / 8; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
  auto move_max = [&](int half, float x) {       // the running max is at least x from here on
    if (x > m[half]) {
      const float a = ptx::ex2(m[half] - x);
      l[half] *= a;
#pragma unroll
      for (int j = 0; j < D / 8; ++j) o[j][2 * half] *= a, o[j][2 * half + 1] *= a;
      m[half] = x;
    }
  };

  // The drafted tokens first: they need nothing of the kernel before. Without a tree no row of the block looks past its last token.
  if (L.d.k_new && block0 / L.d.gq < drafted) {
    const int last = min(block0 + (kTileWarps / wpr) * 16, L.rows) - 1;
    const int end = L.d.tree ? drafted : min(drafted, last / L.d.gq + 1);
    const uint16_t* qb = static_cast<const uint16_t*>(L.d.q) + b * L.d.qs[0] + h * L.d.gq * L.d.qs[2];
    uint32_t qf[D / 16][4];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const uint32_t* q = reinterpret_cast<const uint32_t*>(qb + t[half] * L.d.qs[1] + (in[half] ? r[half] % L.d.gq : 0) * L.d.qs[2] + fc);
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        qf[ks][half] = live[half] ? __ldg(q + ks * 8) : 0u;
        qf[ks][half + 2] = live[half] ? __ldg(q + ks * 8 + 4) : 0u;
      }
    }
    const uint32_t kt = ptx::smem_addr(tile), vt = kt + KB * BLOCK;
    for (int c0 = 0; c0 < end; c0 += kChunk) {
      const int count = min(kChunk, end - c0), padded = (count + 15) & ~15;
      uint64_t bits[2];                          // the allowed keys of the chunk
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (L.d.tree) {
          const int32_t* w = L.d.tree + b * L.d.trs[0] + t[half] * L.d.trs[1] + c0 / 32;
          bits[half] = static_cast<uint32_t>(__ldg(w));
          if (count > 32) bits[half] |= static_cast<uint64_t>(static_cast<uint32_t>(__ldg(w + 1))) << 32;
        } else {
          bits[half] = t[half] - c0 >= 63 ? ~0ull : t[half] < c0 ? 0ull : (2ull << (t[half] - c0)) - 1ull;
        }
        if (count < 64) bits[half] &= (1ull << count) - 1ull;
        if (!live[half]) bits[half] = 0;
      }
      if (c0 > 0) __syncthreads();
      bool bad = false;
      for (int i = threadIdx.x; i < padded * (D / 8); i += 32 * kTileWarps) {
        const int row = i / (D / 8), ch = i % (D / 8);
        uint4 k = make_uint4(0, 0, 0, 0), v = k;
        if (row < count) {
          const int64_t tok = c0 + row;
          k = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(L.d.k_new) + b * L.d.kns[0] + tok * L.d.kns[1] + h * L.d.kns[2]) + ch);
          v = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(L.d.v_new) + b * L.d.vns[0] + tok * L.d.vns[1] + h * L.d.vns[2]) + ch);
        }
        bad = bad || !all_finite<T>(v);
        uint8_t* dst = tile + (ch / 8) * BLOCK + row * 128 + ((ch & 7) ^ (row & 7)) * 16;
        *reinterpret_cast<uint4*>(dst) = k;
        *reinterpret_cast<uint4*>(dst + KB * BLOCK) = v;
      }
      bad = __syncthreads_or(bad);
      for (int k0 = 16 * wi; k0 < padded; k0 += 16 * wpr) {
        const uint32_t allow[2] = {static_cast<uint32_t>(bits[0] >> k0) & 0xffffu, static_cast<uint32_t>(bits[1] >> k0) & 0xffffu};
        if (!__any_sync(0xffffffffu, (allow[0] | allow[1]) != 0)) continue;
        float p[2][4] = {};
        const int k_row = k0 + (mi >> 1) * 8 + r8, v_row = k0 + (mi & 1) * 8 + r8;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          uint32_t kf[4];
          ptx::ldmatrix4(kf, kt + (ks / 4) * BLOCK + k_row * 128 + ((((ks % 4) * 2 + (mi & 1)) ^ r8) << 4));
          ptx::mma16816<T>(p[0], qf[ks], kf[0], kf[1]);
          ptx::mma16816<T>(p[1], qf[ks], kf[2], kf[3]);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          float top = -INFINITY;
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float& x = p[j][2 * half + e];
              x = (allow[half] >> (j * 8 + fc + e)) & 1 ? x * L.d.scale_log2 : -INFINITY;
              top = fmaxf(top, x);
            }
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          move_max(half, top - kHeadroom);
          const float ref = m[half] == -INFINITY ? 0.f : m[half];
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float& x = p[j][2 * half + e];
              x = ptx::ex2(x - ref);
              l[half] += x;
            }
        }
        if (!bad) {
          const uint32_t pa[4] = {T::pack(p[0][0], p[0][1]), T::pack(p[0][2], p[0][3]), T::pack(p[1][0], p[1][1]), T::pack(p[1][2], p[1][3])};
#pragma unroll
          for (int j = 0; j < D / 16; ++j) {
            uint32_t vf[4];
            ptx::ldmatrix4_t(vf, vt + (j / 4) * BLOCK + v_row * 128 + ((((j % 4) * 2 + (mi >> 1)) ^ r8) << 4));
            ptx::mma16816<T>(o[2 * j], pa, vf[0], vf[1]);
            ptx::mma16816<T>(o[2 * j + 1], pa, vf[2], vf[3]);
          }
        } else {
#pragma unroll 1
          for (int src = 0; src < 4; ++src)      // the lane of the quad that holds the weight
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int half = i & 1, e = (i >> 1) & 1, j8 = (i >> 2) * 8, key = j8 + 2 * src + e;
              const float w = __shfl_sync(0xffffffffu, p[i >> 2][2 * half + e], (lane & ~3) | src);
              if ((allow[half] >> key) & 1)
#pragma unroll
                for (int j = 0; j < D / 8; ++j) {
                  const uint32_t v = *reinterpret_cast<const uint32_t*>(tile + (KB + j / 8) * BLOCK + (k0 + key) * 128 +
                                                                        ((j % 8) ^ (key & 7)) * 16 + fc * 2);
                  o[j][2 * half] = fmaf(w, T::lo(v), o[j][2 * half]);
                  o[j][2 * half + 1] = fmaf(w, T::hi(v), o[j][2 * half + 1]);
                }
            }
        }
      }
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      l[half] += __shfl_xor_sync(0xffffffffu, l[half], 1);
      l[half] += __shfl_xor_sync(0xffffffffu, l[half], 2);
    }
  }

  ptx::grid_wait();
  ptx::grid_launch_next();
  if (tiles > 0) {
    int n[2];                                    // partials of this warp
    int64_t row0[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int slot = r[half] / L.slot_rows, rt = slot / L.slots;
      const int in_slot = L.wide && !L.qt.head_inner ? (r[half] % L.d.gq) * L.qt.tokens + t[half] % L.qt.tokens : r[half] % L.slot_rows;
      const int row = (slot % L.slots) * (L.tile_rows / L.slots) + in_slot;
      const int u0 = first + rt * uc.units(tiles) + uc.lead;
      const int i0 = split_owner(u0, sp.total, ctas), i1 = split_owner(u0 + tiles - 1, sp.total, ctas);
      n[half] = live[half] ? (i1 - i0 + 1 - wi + wpr - 1) / wpr : 0;
      row0[half] = static_cast<int64_t>(i0 + bh * L.row_tiles + rt + wi) * L.tile_rows + row;
    }
    const int64_t step = static_cast<int64_t>(wpr) * L.tile_rows;
    for (int i = 0; i < max(n[0], n[1]); ++i) {
      float2 x[2], y[2][D / 8];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const bool has = i < n[half];
        const int64_t at = row0[half] + i * step;
        x[half] = has ? L.part_ml[at] : make_float2(-INFINITY, 0.f);
        const float2* src = reinterpret_cast<const float2*>(L.part_o + at * D + fc);
#pragma unroll
        for (int j = 0; j < D / 8; ++j) y[half][j] = has ? src[4 * j] : make_float2(0.f, 0.f);
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        move_max(half, x[half].x);
        const float w = ptx::ex2(x[half].x - (m[half] == -INFINITY ? 0.f : m[half]));
        l[half] = fmaf(w, x[half].y, l[half]);
#pragma unroll
        for (int j = 0; j < D / 8; ++j) {
          o[j][2 * half] = fmaf(w, y[half][j].x, o[j][2 * half]);
          o[j][2 * half + 1] = fmaf(w, y[half][j].y, o[j][2 * half + 1]);
        }
      }
    }
  }
  if (wpr > 1) {
    if ((lane & 3) == 0) join_ml[warp][fr] = make_float2(m[0], l[0]), join_ml[warp][fr + 8] = make_float2(m[1], l[1]);
    __syncthreads();                             // (the chunk's last readers are done too)
    float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      for (int w = 0; w < wpr; ++w) top[half] = fmaxf(top[half], join_ml[group * wpr + w][fr + 8 * half].x);
      const float ref = top[half] == -INFINITY ? 0.f : top[half];
      for (int w = 0; w < wpr; ++w) {
        const float2 x = join_ml[group * wpr + w][fr + 8 * half];
        sum[half] = fmaf(x.y, ptx::ex2(x.x - ref), sum[half]);
      }
      const float f = ptx::ex2(m[half] - ref);
#pragma unroll
      for (int j = 0; j < D / 8; ++j) o[j][2 * half] *= f, o[j][2 * half + 1] *= f;
      m[half] = top[half];
      l[half] = sum[half];
    }
    float4* join = reinterpret_cast<float4*>(tile) + group * (wpr - 1) * (D / 8) * 32 + lane;
    static_assert((kTileWarps - 1) * (D / 8) * 32 * 16 <= 2 * KB * BLOCK, "three warps' O");
    if (wi > 0)
#pragma unroll
      for (int j = 0; j < D / 8; ++j) join[((wi - 1) * (D / 8) + j) * 32] = make_float4(o[j][0], o[j][1], o[j][2], o[j][3]);
    __syncthreads();
    if (wi > 0) return;
    for (int w = 0; w < wpr - 1; ++w)
#pragma unroll
      for (int j = 0; j < D / 8; ++j) {
        const float4 x = join[(w * (D / 8) + j) * 32];
        o[j][0] += x.x, o[j][1] += x.y, o[j][2] += x.z, o[j][3] += x.w;
      }
  }
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (!in[half]) continue;
    const int head = h * L.d.gq + r[half] % L.d.gq;
    const float inv = l[half] != 0.f ? 1.f / l[half] : 0.f;  // (a NaN sum stays one)
    uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(L.o) +
                                                ((static_cast<int64_t>(b) * L.d.tokens + t[half]) * L.d.hq + head) * D + fc);
#pragma unroll
    for (int j = 0; j < D / 8; ++j) dst[4 * j] = T::pack(o[j][2 * half] * inv, o[j][2 * half + 1] * inv);
    if ((lane & 3) == 0)
      L.lse[(static_cast<int64_t>(head) * L.c.batch + b) * L.d.tokens + t[half]] = row_lse<T>(m[half], l[half]);
  }
}

template <class T, int D, int MG>
cudaError_t launch_few(const CacheAttnLaunch& L, cudaStream_t stream) {
  using C = FewCfg<D, MG>;
  static_assert(C::SMEM <= 232448, "shared memory budget");
  auto kern = cache_attn_few_kernel<T, D, MG>;
  static PerDeviceAttr once;
  const cudaError_t e = raise_smem_limit(once, reinterpret_cast<const void*>(kern), C::SMEM);
  if (e != cudaSuccess) return e;
  return launch_after(kern, dim3(L.n_ctas), C::THREADS, C::SMEM, stream, L);
}

template <class T, int D>
cudaError_t launch_d(const CacheAttnLaunch& L, cudaStream_t stream) {
  cudaError_t e;
  if (L.wide) e = launch_cache_attn_wide(L, stream);
  else if (D == 128 || L.tile_rows == 16) e = launch_few<T, D, 1>(L, stream);
  else e = launch_few<T, 64, 2>(L, stream);
  if (e != cudaSuccess) return e;
  if (L.join_tile) {
    const int per_block = 16 * (kTileWarps / L.join_warps);
    return launch_after(cache_join_tile_kernel<T, D>, dim3((L.rows + per_block - 1) / per_block, L.c.batch * L.c.hkv),
                        32 * kTileWarps, 0, stream, L, L.join_warps);
  }
  const int per = kJoinWarps / L.join_warps;
  return launch_after(cache_join_kernel<T, D>, dim3((L.rows + per - 1) / per, L.c.batch * L.c.hkv), 32 * kJoinWarps, 0, stream,
                      L, L.join_warps);
}

}  // namespace

// Few rows a CTA or many. A few-rows CTA starts faster and its partials are 16 or
// 32 rows high; but every 16 rows read the keys again, which the wide one does
// once for 128 or 256. By the units of 64 keys times 16 rows that the capacity
// of the tables allows, us with few / wide: 7 heads a KV head of 128, one
// sequence of 8,192 with 6 tokens (1,536 units) 14.5 / 15.8, 16,384 with 3
// (2,048) 14.7 / 19.0, 32,768 with 4 (4,096) 19.6 / 22.8, with 6 (6,144) 23.5 / 23.2,
// with 12 (12,288) 36.6 / 24.8; 32 of 4,096 with 3 (16,384) 74 / 54. Rows 17 to
// 32 of heads of 64 have a tile of their own: 32,768 tokens and 8 KV heads take 28.5 us
// in tiles of 16, 22.3 in one of 32 and 27.1 wide; below 2,048 units 16 is faster
// (2,048 tokens: 8.6 / 9.9).
// At least three units a CTA, wide two, for fewer partials in the join: one drafted token
// over 4,160 takes 9.8 us with one, 9.5 with two, 9.1 with three and 9.6 with four (8,192: 12.2, 9.7, 10.4,
// 10.6; one KV head over 16,384: 13.7, 11.3, 10.4, 10.5); 24 over 4,160, wide, 22.6, 18.9 and 20.3 with three.
// The lead stands for what a problem costs beside its keys: 200 sequences of 64 take 26.7 us
// without and 24.3 with two units (few), 8 of 2,048 with 24 tokens 33.5 and 32.4 with one (wide).
CacheAttnShape cache_attn_shape(int rows, int tokens, int64_t problems, int64_t capacity, int head_dim, const QueryTile& qt,
                                bool q_map, int n_sm) {
  CacheAttnShape s;
  const int64_t units = (capacity + kKeys - 1) / kKeys * problems * ((rows + 15) / 16);
  const bool tall = head_dim == 64 && rows > 16 && units > 14 * n_sm;
  if (rows > 16 && units > 28 * n_sm && q_map && !(tall && rows <= 32)) {
    s.wide = true;
    s.slot_rows = qt.rows;
    const int slots = (rows + s.slot_rows - 1) / s.slot_rows;
    s.slots = slots > 1 ? 2 : 1;
    s.tile_rows = 128 * s.slots;
    s.row_tiles = (slots + s.slots - 1) / s.slots;
    s.key_tile = 128;
    s.n_ctas = n_sm;
    s.min_units = 2;
    s.lead = 1;
  } else {
    s.wide = false;
    s.slots = 1;
    s.slot_rows = s.tile_rows = tall ? 32 : 16;
    s.row_tiles = (rows + s.tile_rows - 1) / s.tile_rows;
    s.key_tile = kKeys;
    s.n_ctas = 2 * n_sm;
    s.min_units = 3;
    s.lead = 2;
  }
  // Warps that share a row in the join: each has four partials or more, and the
  // blocks are not many more than fit. One drafted token over 32,768: 20.8 us with one
  // warp, 14.6 with eight; 64 sequences of 300: 15.2 with one, 25.4 with eight; 24 drafted
  // tokens over 4,160: 30.3 with one, 22.4 with four, 23.9 with eight.
  const int64_t all_rows = problems * rows, tiles = (capacity + s.key_tile - 1) / s.key_tile;
  const int64_t partials = std::min<int64_t>(s.n_ctas / (problems * s.row_tiles), tiles / s.min_units);
  // A tile of rows or row by row: by the rows' products with drafted tokens. The whole call, tile / row by row: 64
  // sequences of 256 with 64 tokens (7.3 million) 108 / 377 us, 8 of 4,096 with 24 (129,024) 36.6 / 39.2, one of 4,160 with 64
  // (114,688) 33.7 / 33.0, 8 with 12 (32,256) 29.6 / 26.8. Fewer rows are shared by more warps: 5,376 by four
  // 36.6 us, by one 42.2; 43,008 by four 87, by one 46.3.
  s.join_tile = all_rows * tokens > 49152;
  s.join_warps = s.join_tile ? 4 : 8;
  while (s.join_warps > 1 && (partials < s.join_warps * (s.join_tile ? 1 : 4) || all_rows * s.join_warps > (s.join_tile ? 24576 : 4096)))
    s.join_warps /= 2;
  return s;
}

cudaError_t launch_cache_attn(const CacheAttnLaunch& L, cudaStream_t stream) {
  if (L.c.dtype == 0) return L.c.head_dim == 128 ? launch_d<BF16, 128>(L, stream) : launch_d<BF16, 64>(L, stream);
  return L.c.head_dim == 128 ? launch_d<FP16, 128>(L, stream) : launch_d<FP16, 64>(L, stream);
}

}  // namespace evisel
