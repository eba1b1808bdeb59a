// Attention of drafted tokens over a paged cache: partial results of ranges of
// cached keys, and their join with the drafted tokens' own attention.
//
//   s_rm = scale q_r . k_m,  O_r = sum_m exp(s_rm - LSE_r) v_m
//
// over a (sequence, KV head)'s rows r = (token, head of the group).
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
        // Running max (log2 units), moved only when it grows by more than 2^8.
        float tm[MG][2];
        bool grows = false;
#pragma unroll
        for (int g = 0; g < MG; ++g)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            float x = fmaxf(fmaxf(sc[g][0][2 * half], sc[g][0][2 * half + 1]), fmaxf(sc[g][1][2 * half], sc[g][1][2 * half + 1]));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
            tm[g][half] = x * L.d.scale_log2;
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
// max of its own.
constexpr int kJoinWarps = 8;

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
    L.lse[(static_cast<int64_t>(head) * L.c.batch + b) * L.d.tokens + t] = l != 0.f ? (m + __log2f(l)) * kLn2 : -INFINITY;
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
  const cudaError_t e = L.wide               ? launch_cache_attn_wide(L, stream)
                        : L.tile_rows == 16 ? launch_few<T, D, 1>(L, stream)
                                            : launch_few<T, D, 2>(L, stream);
  if (e != cudaSuccess) return e;
  // Warps per row: as many as keep the rows' blocks within about two per SM.
  const int64_t rows = static_cast<int64_t>(L.c.batch) * L.c.hkv * L.rows;
  const int wpr = rows >= 2048 ? 1 : rows >= 1024 ? 2 : rows >= 512 ? 4 : 8;
  const int per = kJoinWarps / wpr;
  return launch_after(cache_join_kernel<T, D>, dim3((L.rows + per - 1) / per, L.c.batch * L.c.hkv), 32 * kJoinWarps, 0, stream,
                      L, wpr);
}

}  // namespace

CacheAttnShape cache_attn_shape(int rows, const QueryTile& qt, bool q_map, int n_sm) {
  CacheAttnShape s;
  if (rows > 32 && q_map) {
    s.wide = true;
    s.slot_rows = qt.rows;
    const int slots = (rows + s.slot_rows - 1) / s.slot_rows;
    s.slots = slots > 1 ? 2 : 1;
    s.tile_rows = 128 * s.slots;
    s.row_tiles = (slots + s.slots - 1) / s.slots;
    s.key_tile = 128;
    s.n_ctas = n_sm;
    s.min_units = 1;
    s.lead = 1;
    return s;
  }
  s.wide = false;
  s.slots = 1;
  s.slot_rows = s.tile_rows = rows <= 16 ? 16 : 32;
  s.row_tiles = (rows + s.tile_rows - 1) / s.tile_rows;
  s.key_tile = kKeys;
  s.n_ctas = 2 * n_sm;
  s.min_units = 3;
  s.lead = 2;
  return s;
}

cudaError_t launch_cache_attn(const CacheAttnLaunch& L, cudaStream_t stream) {
  if (L.c.dtype == 0) return L.c.head_dim == 128 ? launch_d<BF16, 128>(L, stream) : launch_d<BF16, 64>(L, stream);
  return L.c.head_dim == 128 ? launch_d<FP16, 128>(L, stream) : launch_d<FP16, 64>(L, stream);
}

}  // namespace evisel
