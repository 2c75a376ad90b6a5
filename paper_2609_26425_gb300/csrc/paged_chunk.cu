// paged_chunk.cu -- attention of many rows of a sequence over its pages: chunks
// and prompts.
//
// Mathematics: as in paged_step.cu, with the rows of a sequence ordered (Query
// token, grouped head), so that the grouped heads of a token share every K and
// V tile.  The bound is the tensor pipe: 4 D operations per visible (row, key).
//
// A CTA takes 256 rows as two tiles of 128 (the M of tcgen05) over a common list
// of 128-key tiles: S_i = Q_i K^T goes to TMEM, a warpgroup per tile turns it
// into P (thread = row) written over S as 16-bit pairs, and P V accumulates in
// TMEM with P read from there.  P is rounded to the cache's type because the MMA takes
// both factors in one type, and P in two parts would cost half as many MMAs again;
// its sum l is taken before the rounding.  The error against 64 bits is 1.4 times the
// fp32 form's (2.3e-3 against 1.7e-3 in bf16, most of that the result's own rounding).  Two tiles, because the softmax of one then runs
// beside the MMAs of the other.  TMEM: S0 | S1 | O0 | O1.
// The chain S, softmax, P V, next S sets the pace, so the row maximum is kept off
// it: P is taken against the maximum known before the tile, one pass over S with
// the exponentials (32 a cycle and SM) as its only bound.  P, l and O are
// floating-point multiples of the same power of two, so a maximum that has grown
// costs nothing until P has grown by 2^kTau; a half tile whose sum is above that
// (no P above it can hide in a smaller sum) is taken again against its rows' new
// maxima.
// Few rows over many keys are split along the keys; the parts' O, m and l go
// through global memory to a second kernel over all SMs, launched ahead so that
// it stands ready.  (A join by a group's last CTA took 11 us of 69 at 880 Queries
// x 12 heads: one SM reads 384 KB at 42 bytes a cycle.  Parts as clusters joined
// through shared memory: 46 clusters of 3 fit where 48 were wanted, 97 us.)
// Warps: four per row tile softmax, then MMA issue, a TMA producer each for K and
// V (a 16-token page is a copy of 2 KB: one warp's issue rate would bound the
// tile), and the Values' guard.
// The guard clears the Values of keys that no row of the CTA sees (0 x inf is
// not 0 in the MMA) in the tiles at the edges of the mask, and waves the others
// through; infinities and NaN in Values that some rows see and others do not
// are taken out of the product and added to the rows that see them at the end.
#include <type_traits>

#include "paged.cuh"

namespace qwm {
namespace {
using namespace ptx;

constexpr int TK = 128;
constexpr int ST = 2;                     // K tiles and V tiles in flight
constexpr int BLK = 16384;                // 128 rows x 128 bytes

enum { B_KFULL = 0, B_KEMPTY = 2, B_VFULL = 4, B_VRDY = 6, B_VEMPTY = 8, B_SFULL = 10, B_QRDY = 12, B_PV = 14,
       B_PFULL = 16 /* tile, half */, B_OFIN = 20 };

constexpr int NQ = 2, ROWS = 128 * NQ;               // row tiles and rows of a CTA
constexpr int W_MMA = 4 * NQ, W_K = W_MMA + 1, W_V = W_MMA + 2;  // W_MMA + 3: the guard
constexpr int NT = (4 * NQ + 4) * 32;

template <int D>
struct Smem {
  static constexpr int NB = D / 64;                  // 64-channel blocks of a tile
  static constexpr int Q = 0;                        // tile i, block k at (i * NB + k) * BLK
  static constexpr int K = NQ * NB * BLK;            // stage s, block k at (s * NB + k) * BLK
  static constexpr int V = K + ST * NB * BLK;
  static constexpr int BAR = V + ST * NB * BLK;
  static constexpr int TOTAL = BAR + 256 + 1024;
};

__device__ __forceinline__ void umma_ss_e(uint32_t d, uint64_t ad, uint64_t bd, uint32_t id, uint32_t acc, uint32_t e) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(ad), "l"(bd), "r"(id), "r"(acc), "r"(e)
      : "memory");
}
__device__ __forceinline__ void umma_ts_e(uint32_t d, uint32_t at, uint64_t bd, uint32_t id, uint32_t acc, uint32_t e) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(at), "l"(bd), "r"(id), "r"(acc), "r"(e)
      : "memory");
}
__device__ __forceinline__ void commit_e(uint32_t bar, uint32_t e) {
  asm volatile(
      "{\n\t.reg .pred q;\n\t"
      "setp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(e)
      : "memory");
}

// Bits [a, b) of a 32-bit word (any a <= b, also outside 0..32).
__device__ __forceinline__ uint32_t bits(int a, int b) {
  const uint32_t hi = b <= 0 ? 0u : (b >= 32 ? 0xFFFFFFFFu : (1u << b) - 1u);
  const uint32_t lo = a <= 0 ? 0u : (a >= 32 ? 0xFFFFFFFFu : (1u << a) - 1u);
  return hi & ~lo;
}

constexpr float pow2(int e) { return e > 0 ? 2.0f * pow2(e - 1) : (e < 0 ? 0.5f * pow2(e + 1) : 1.0f); }
// Natural-log sum-exp of a row: `m` is the power that its P were taken against, l
// their sum.  -inf (and log 0) where nothing was seen, NaN with a NaN sum.
template <typename T>
__device__ __forceinline__ float log_sum(float m, float l) {
  return (m - (float)Elem<T>::kBias + log2f(l * pow2(Elem<T>::kBias))) * 0.69314718055994531f;
}

template <typename T, int D>
__global__ void __launch_bounds__(NT, 1) paged_chunk(const __grid_constant__ CUtensorMap map, const PagedArgs a) {
  using L = Smem<D>;
  constexpr int NB = L::NB;
  extern __shared__ uint8_t raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  __shared__ uint32_t s_tmem;
  __shared__ int s_err, s_poison;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  auto bar = [&](int i) { return smem_u32(sm + L::BAR) + 8u * i; };
  if (tid == 0) {
    for (int s = 0; s < 2; ++s) {
      mbar_init(bar(B_KFULL + s), 1);
      mbar_init(bar(B_KEMPTY + s), 1);
      mbar_init(bar(B_VFULL + s), 1);
      mbar_init(bar(B_VRDY + s), 1);
      mbar_init(bar(B_VEMPTY + s), 1);
      mbar_init(bar(B_SFULL + s), 1);
      mbar_init(bar(B_PV + s), 1);
      mbar_init(bar(B_PFULL + 2 * s), 4);
      mbar_init(bar(B_PFULL + 2 * s + 1), 4);
      mbar_init(bar(B_QRDY + s), 4);
    }
    mbar_init(bar(B_OFIN), 1);
    s_err = 0;
    s_poison = 0;
    fence_mbar_init();
  }
  grid_begin();
  const int b = blockIdx.z, hk = blockIdx.y;
  const int rtiles = gridDim.x / a.nsplit;
  // the row tiles with the most keys first
  const int rt = rtiles - 1 - (int)(blockIdx.x % rtiles), part = blockIdx.x / rtiles;
  Seq sq;
  if (!load_seq(a, b, sq) && blockIdx.x == 0 && hk == 0 && tid == 0) record_status(a.status, QWM_ERR_INVALID_ARG);
  const int64_t rows = (int64_t)sq.qn * a.G;
  const int64_t r0 = (int64_t)rt * ROWS;
  if (r0 >= rows) return;
  const int nrow = (int)min((int64_t)ROWS, rows - r0);
  const int nqt = nrow > 128 ? 2 : 1;
  const int p0 = sq.kv - sq.qn;                       // token of the sequence's first row
  // row r0 + i is new token tokA + (remA + i) / G, grouped head (remA + i) % G
  const int tokA = (int)(r0 / a.G);
  const uint32_t G = (uint32_t)a.G, remA = (uint32_t)(r0 - (int64_t)tokA * a.G);
  const int tokB = tokA + (int)((remA + (uint32_t)nrow - 1) / G);
  const Tiles tl = make_tiles<TK>(p0 + tokA, p0 + tokB, sq.kv, a.block, a.window, a.sinks);
  const int per = max((tl.n + a.nsplit - 1) / a.nsplit, a.min_tiles);
  const int parts = max(1, (tl.n + per - 1) / per);
  if (part >= parts) return;
  const int t0 = part * per, n = max(0, min(tl.n, t0 + per) - t0);   // this part's tiles: t0 .. t0 + n - 1

  auto wait_all = [&](int i, uint32_t ph) -> bool {
    return __all_sync(0xFFFFFFFFu, mbar_wait(bar(i), ph, a.wait_ns));
  };
  __syncthreads();                                    // the barriers are set up
  if (warp == W_MMA) {
    tmem_alloc(smem_u32(&s_tmem), 512);
    tmem_relinquish();
  }
  if (warp < W_MMA && (warp >> 2) < nqt) {
    const int i = warp >> 2;
    // Q_i: each warp its 32 rows, a row's 16-byte chunks over neighbouring lanes
    uint8_t* sQ = sm + L::Q + i * NB * BLK;
    constexpr int CH = D / 8;
    {
      uint4 v[CH];
#pragma unroll
      for (int k = 0; k < CH; ++k) {
        const int idx = k * 32 + lane, rr = (warp & 3) * 32 + idx / CH, c = idx % CH;
        const uint32_t r = remA + min(i * 128 + rr, nrow - 1);
        v[k] = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + (sq.q0 + tokA + r / G) * a.q_tok +
                                               (hk * a.G + (int)(r % G)) * a.q_head + c * 8);
      }
#pragma unroll
      for (int k = 0; k < CH; ++k) {
        const int idx = k * 32 + lane, rr = (warp & 3) * 32 + idx / CH, c = idx % CH;
        if (i * 128 + rr >= nrow) v[k] = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(sQ + (c >> 3) * BLK + rr * 128 + (((c & 7) ^ (rr & 7)) << 4)) = v[k];
      }
    }
    fence_proxy_async_smem();
  }
  // The producers and the guard touch no TMEM: their first copies go out while it is
  // being allocated and the Queries come in.  (All warps waiting for the allocation
  // and the Queries loaded after it: 880 Queries x 12 heads 64.0 us against 62.5;
  // three ragged prompts of 64 channels 79.5 against 80.5.)
  uint32_t tbase = 0;
  if (warp <= W_MMA) {
    tc_fence_before();
    named_bar_sync(1, (W_MMA + 1) * 32);
    tc_fence_after();
    tbase = s_tmem;
  }
  const float sl2 = a.scale * 1.4426950408889634f;

  if (warp < W_MMA) {
    // ------------------------------------------------------------ softmax
    const int i = warp >> 2, row = tid & 127;
    if (i < nqt) {
      uint8_t* sQ = sm + L::Q + i * NB * BLK;
      constexpr int CH = D / 8;
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_QRDY + i));

      const bool has = i * 128 + row < nrow;
      const int tok = has ? tokA + (int)((remA + i * 128 + row) / G) : tokB;
      const int head = hk * a.G + (has ? (int)((remA + i * 128 + row) % G) : 0);
      const Span sp = has ? row_span(p0 + tok, sq.kv, a.block, a.window) : Span{0, 0};
      const uint32_t lrow = (uint32_t)((warp & 3) * 32) << 16;
      const uint32_t tS = tbase + 128 * i + lrow, tO = tbase + 128 * NQ + D * i + lrow;
      float m_run = has ? -INFINITY : 0.0f, l_run = 0.0f;
      const uint64_t SL = f2pack(sl2, sl2);
      constexpr float kMost = pow2(Elem<T>::kTau - Elem<T>::kBias);
      // P = 2^(s sl2 - power(m_run))
      auto power = [&](float m) { return fmaf(m, sl2, (float)Elem<T>::kBias); };
      // Raises every row of the warp to its own maximum, and O with it (the P V
      // before it are complete)
      auto raise = [&](float mt, bool rescale) {
        const float alpha = mt > m_run ? ex2f(power(m_run) - power(mt)) : 1.0f;
        m_run = fmaxf(m_run, mt);
        l_run *= alpha;
        if (rescale) {
#pragma unroll 1
          for (int cb = 0; cb < D / 16; ++cb) {
            uint32_t t[16];
            tmem_ld16(tO + cb * 16, t);
#pragma unroll
            for (int e = 0; e < 16; ++e) t[e] = __float_as_uint(__uint_as_float(t[e]) * alpha);
            tmem_st16(tO + cb * 16, t);
          }
        }
      };
      bool ok = true;
      for (int jt = 0; jt < n; ++jt) {
        if (!(ok = wait_all(B_SFULL + i, jt & 1))) break;
        tc_fence_after();
        const int j0 = tile_at(tl, t0 + jt) * TK;
        const bool open = __all_sync(0xFFFFFFFFu, !has || (j0 + TK <= sp.hi && (j0 >= sp.lo || j0 + TK <= a.sinks)));
        // Which keys of each 32-key block this row sees; a warp whose rows all
        // see a whole block, or none of it, takes it without the selection.
        enum { kNone, kSome, kAll };
        auto seen = [&](int blk, uint32_t& see) -> int {
          see = 0xFFFFFFFFu;
          const int c = j0 + 32 * blk;
          if (has) see = bits(sp.lo - c, sp.hi - c) | bits(-c, min(a.sinks, sp.hi) - c);
          return __all_sync(0xFFFFFFFFu, see == 0xFFFFFFFFu) ? kAll : (__any_sync(0xFFFFFFFFu, has && see != 0) ? kSome : kNone);
        };
        auto select = [&](uint32_t (&w)[32], uint32_t see) {
#pragma unroll
          for (int e = 0; e < 32; ++e) w[e] = (see >> e) & 1 ? w[e] : 0xFF800000u;
        };
        // where a row has no maximum yet, the tile's comes first
        if (__any_sync(0xFFFFFFFFu, m_run == -INFINITY)) {
          float mt = -INFINITY;
          if (open) {
            mt = tmem_max128(tS);
          } else {
#pragma unroll
            for (int blk = 0; blk < 4; ++blk) {
              uint32_t see, w[32];
              const int kind = seen(blk, see);
              if (kind == kNone) continue;
              tmem_ld32_start(tS + 32 * blk, w);
              tmem_ld32_wait(w);
              if (kind == kSome) select(w, see);
#pragma unroll
              for (int e = 0; e < 32; e += 2) mt = fmax3f(mt, __uint_as_float(w[e]), __uint_as_float(w[e + 1]));
            }
          }
          if (__any_sync(0xFFFFFFFFu, mt > m_run)) raise(mt, jt > 0);
        }
        // One pass over S in two halves of 64 keys, each handed on as soon as it is
        // done: P against m_run, and its sum.
        uint32_t pk[32];
        uint64_t sum, MB;
        auto begin_half = [&]() {
          const float mb = m_run == -INFINITY ? 0.0f : power(m_run);
          MB = f2pack(-mb, -mb);
          sum = f2pack(0.0f, 0.0f);
        };
        auto block = [&](auto masked, int blk, uint32_t (&w)[32]) {
          if (masked) {
            uint32_t see;
            const int kind = seen(blk, see);
            if (kind == kNone) {
#pragma unroll
              for (int e = 0; e < 16; ++e) pk[16 * (blk & 1) + e] = 0u;
              return;
            }
            if (kind == kSome) select(w, see);
          }
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float s0 = __uint_as_float(w[e]), s1 = __uint_as_float(w[e + 1]);
            float x, y;
            f2unpack(fma2(f2pack(s0, s1), SL, MB), x, y);
            x = ex2f(x);
            y = ex2f(y);
            sum = add2(sum, f2pack(x, y));
            pk[16 * (blk & 1) + (e >> 1)] = Elem<T>::pack(x, y);
          }
        };
        auto pass = [&](auto masked) {
          uint32_t v[2][32];
          tmem_ld32_start(tS, v[0]);
#pragma unroll
          for (int blk = 0; blk < 4; ++blk) {
            tmem_ld32_wait(v[blk & 1]);
            if (blk < 3) tmem_ld32_start(tS + 32 * (blk + 1), v[(blk + 1) & 1]);
            if ((blk & 1) == 0) begin_half();
            block(masked, blk, v[blk & 1]);
            if ((blk & 1) == 0) continue;
            const int half = blk >> 1;
            float sx, sy;
            f2unpack(sum, sx, sy);
            if (__any_sync(0xFFFFFFFFu, sx + sy > kMost)) {
              // again against the new maximum; the first half's P V has to be in O
              // before O is scaled for the second's
              if (half == 1) {
                if (!(ok = wait_all(B_PV + i, jt & 1))) return;
                tc_fence_after();
              }
              uint32_t u[32];
              float mt = -INFINITY;
#pragma unroll 1
              for (int k = 0; k < 2; ++k) {
                uint32_t see;
                const int kind = seen(2 * half + k, see);
                tmem_ld32_start(tS + 64 * half + 32 * k, u);
                tmem_ld32_wait(u);
                if (kind == kNone) continue;
                if (kind == kSome) select(u, see);
#pragma unroll
                for (int e = 0; e < 32; e += 2) mt = fmax3f(mt, __uint_as_float(u[e]), __uint_as_float(u[e + 1]));
              }
              raise(mt, half == 1 || jt > 0);
              begin_half();
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                tmem_ld32_start(tS + 64 * half + 32 * k, u);
                tmem_ld32_wait(u);
                block(std::true_type{}, 2 * half + k, u);
              }
              f2unpack(sum, sx, sy);
            }
            l_run += sx + sy;
            tmem_st16(tS + 32 * half, *reinterpret_cast<uint32_t(*)[16]>(pk));
            tmem_st16(tS + 32 * half + 16, *reinterpret_cast<uint32_t(*)[16]>(pk + 16));
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(B_PFULL + 2 * i + half));
          }
        };
        if (open) pass(std::false_type{});
        else pass(std::true_type{});
        if (!ok) break;
      }
      if (ok && n > 0) ok = wait_all(B_OFIN, 0);
      if (!ok) s_err = 1;
      if (ok) {
        tc_fence_after();
        const int64_t group = ((int64_t)b * a.Hk + hk) * rtiles + rt;
        const int64_t pr = (group * a.nsplit + part) * ROWS + i * 128 + row;
        const float inv = l_run > 0.0f || l_run != l_run ? 1.0f / l_run : 0.0f;
        const bool poison = *(volatile int*)&s_poison != 0;
#pragma unroll 1
        for (int cb = 0; cb < D / 32; ++cb) {
          const int c0 = cb * 32;
          float v[32];
          if (n > 0) {
            tmem_ld32(tO + cb * 32, v);
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = 0.0f;
          }
          if (poison && has) {
            // the Values that the guard took out: this row's share of them
            for (int jt = 0; jt < n; ++jt) {
              const int j0 = tile_at(tl, t0 + jt) * TK;
              if (all_see(tl, j0, j0 + TK, a.sinks)) continue;
              for (int j = j0; j < j0 + TK; ++j) {
                if (!sees(j, sp.lo, sp.hi, a.sinks) || all_see(tl, j, j + 1, a.sinks)) continue;
                const int64_t page = a.table[(int64_t)b * a.table_stride + (j >> a.page_log2)];
                if (page < 0 || page >= a.num_pages) continue;
                const T* src = static_cast<const T*>(a.pages) +
                               ((((page * 2 + 1) * a.Hk + hk) << a.page_log2) + (j & ((1 << a.page_log2) - 1))) * D + c0;
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                  const uint32_t w = *reinterpret_cast<const uint32_t*>(src + e);
                  const float2 f = Elem<T>::unpack(w);
                  if ((w & Elem<T>::kExp) == Elem<T>::kExp) v[e] += f.x;
                  if (((w >> 16) & Elem<T>::kExp) == Elem<T>::kExp) v[e + 1] += f.y;
                }
              }
            }
          }
          if (parts == 1) {
            // through Q_i's rows of this warp (every MMA is done), so that the
            // rows leave as whole lines
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int c = cb * 4 + k;
              *reinterpret_cast<uint4*>(sQ + (c >> 3) * BLK + row * 128 + (((c & 7) ^ (row & 7)) << 4)) =
                  make_uint4(Elem<T>::pack(v[8 * k] * inv, v[8 * k + 1] * inv),
                             Elem<T>::pack(v[8 * k + 2] * inv, v[8 * k + 3] * inv),
                             Elem<T>::pack(v[8 * k + 4] * inv, v[8 * k + 5] * inv),
                             Elem<T>::pack(v[8 * k + 6] * inv, v[8 * k + 7] * inv));
            }
          } else if (has) {
            // a part: [channels / 4][row], so that a warp writes whole lines
            float4* d4 = reinterpret_cast<float4*>(a.part_o) + (group * a.nsplit + part) * ROWS * (D / 4) +
                         (int64_t)(c0 / 4) * ROWS + i * 128 + row;
#pragma unroll
            for (int k = 0; k < 8; ++k) d4[k * ROWS] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
          }
        }
        if (parts == 1) {
          __syncwarp();
#pragma unroll 4
          for (int it = 0; it < CH; ++it) {
            const int idx = it * 32 + lane, rr = (warp & 3) * 32 + idx / CH, c = idx % CH;
            if (i * 128 + rr >= nrow) continue;
            const uint32_t r = remA + i * 128 + rr;
            *reinterpret_cast<uint4*>(static_cast<T*>(a.out) + (sq.q0 + tokA + r / G) * a.o_tok +
                                      (int64_t)(hk * a.G + (int)(r % G)) * a.o_head + c * 8) =
                *reinterpret_cast<const uint4*>(sQ + (c >> 3) * BLK + rr * 128 + (((c & 7) ^ (rr & 7)) << 4));
          }
        }
        if (has && parts == 1 && a.lse)
          a.lse[(int64_t)head * a.N + sq.q0 + tok] = log_sum<T>(power(m_run), l_run);
        if (has && parts > 1) a.part_ml[pr] = make_float2(power(m_run), l_run);
      }
    }
  } else if (warp == W_MMA) {
    // ------------------------------------------------------------ MMA issue
    // Order per K/V tile j: P0 V(j) in two halves, S0(j+1), P1 V(j), S1(j+1); S_i(j+1) may
    // overwrite P_i(j) because the MMAs of one thread run in issue order.
    const uint32_t e = elect_one();
    const uint64_t dQ = desc_sw128(smem_u32(sm + L::Q)), dK = desc_sw128(smem_u32(sm + L::K));
    const uint64_t dV = desc_sw128_mn(smem_u32(sm + L::V), BLK);
    auto off = [](int bytes) { return (uint64_t)(bytes >> 4); };
    constexpr uint32_t idS = idesc_f16(128, TK, false, Elem<T>::bf16);
    constexpr uint32_t idPV = idesc_f16(128, D, true, Elem<T>::bf16);
    bool ok = true;
    auto issue_S = [&](int i, int jt) -> bool {
      const int s = jt & 1;
      if (i == 0 && !wait_all(B_KFULL + s, (jt >> 1) & 1)) return false;
      if (jt == 0 && !wait_all(B_QRDY + i, 0)) return false;
      tc_fence_after();
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
          umma_ss_e(tbase + 128 * i, dQ + off((i * NB + kb) * BLK + ks * 32), dK + off((s * NB + kb) * BLK + ks * 32),
                    idS, (kb | ks) != 0, e);
      commit_e(bar(B_SFULL + i), e);
      if (i == nqt - 1) commit_e(bar(B_KEMPTY + s), e);
      return true;
    };
    if (n > 0) {
      for (int i = 0; i < nqt && ok; ++i) ok = issue_S(i, 0);
      for (int jt = 0; jt < n && ok; ++jt) {
        const int s = jt & 1;
        if (!(ok = wait_all(B_VRDY + s, (jt >> 1) & 1))) break;
        for (int i = 0; i < nqt; ++i) {
#pragma unroll
          for (int half = 0; half < 2 && ok; ++half) {
            if (!(ok = wait_all(B_PFULL + 2 * i + half, jt & 1))) break;
            tc_fence_after();
#pragma unroll
            for (int ks = 4 * half; ks < 4 * half + 4; ++ks)
              umma_ts_e(tbase + 128 * NQ + D * i, tbase + 128 * i + 8 * ks, dV + off(s * NB * BLK + ks * 2048), idPV,
                        (jt | ks) != 0, e);
            if (half == 0) commit_e(bar(B_PV + i), e);
          }
          if (!ok) break;
          if (i == nqt - 1) commit_e(bar(B_VEMPTY + s), e);
          if (jt + 1 < n && !(ok = issue_S(i, jt + 1))) break;
        }
      }
      commit_e(bar(B_OFIN), e);
      // the MMAs issued finish before TMEM is freed: the softmax warps, which wait
      // for them as well, may have given up
      if (!mbar_wait(bar(B_OFIN), 0, kDrainNs) || !ok) s_err = 1;
    }
    __syncwarp();
  } else if (warp == W_K || warp == W_V) {
    // ------------------------------------------------------------ producers of K and V
    // lane = box * NB + channel block; a box is the part of a page (at most 64
    // tokens of it) that lies in the tile.  Boxes no row sees are not read.
    const int kv = warp == W_V;
    const int full = kv ? B_VFULL : B_KFULL, empty = kv ? B_VEMPTY : B_KEMPTY;
    const int box_log2 = min(a.page_log2, 6);
    const int boxes = TK >> box_log2;
    const int box = lane / NB, blk = lane % NB;
    const bool mine = box < boxes;
    const int32_t* trow = a.table + (int64_t)b * a.table_stride;
    const uint32_t ring = smem_u32(sm + (kv ? L::V : L::K)) + blk * BLK + ((box << box_log2) * 128);
    auto page_of = [&](int jt, bool& want) -> int {
      const int j0 = tile_at(tl, t0 + jt) * TK + (box << box_log2);
      want = mine && any_sees(tl, j0, j0 + (1 << box_log2), a.sinks);
      return want ? trow[j0 >> a.page_log2] : 0;
    };
    bool want = false, ok = true;
    int page = n > 0 ? page_of(0, want) : 0;
    int jt = 0;
    for (; jt < n && !a.idle; ++jt) {
      const int s = jt & 1;
      bool want_n = false;
      int page_n = 0;
      if (jt + 1 < n) page_n = page_of(jt + 1, want_n);   // its latency runs beside the copies
      if (want && (page < 0 || page >= a.num_pages)) {    // not followed: the first page in its place
        record_status(a.status, QWM_ERR_INVALID_ARG);
        page = 0;
      }
      const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, want)) * (128u << box_log2);
      const int y = (tile_at(tl, t0 + jt) * TK + (box << box_log2)) & ((1 << a.page_log2) - 1);
      if (jt >= ST && !(ok = wait_all(empty + s, ((jt >> 1) - 1) & 1))) break;
      if (lane == 0) mbar_arrive_expect_tx(bar(full + s), bytes);
      __syncwarp();
      if (want) tma_load_3d(ring + s * NB * BLK, &map, blk * 64, y, (page * 2 + kv) * a.Hk + hk, bar(full + s));
      __syncwarp();
      page = page_n;
      want = want_n;
    }
    if (!ok) s_err = 1;
    // the last copies land before the CTA can end: the roles that wait for them may
    // have given up on them
    for (int u = max(0, jt - ST); u < jt; ++u) mbar_wait(bar(full + (u & 1)), (u >> 1) & 1, kDrainNs);
  } else {
    // ------------------------------------------------------------ guard of the Values
    bool ok = true;
    for (int jt = 0; jt < n; ++jt) {
      const int s = jt & 1;
      if (!(ok = wait_all(B_VFULL + s, (jt >> 1) & 1))) break;
      const int j0 = tile_at(tl, t0 + jt) * TK;
      if (!all_see(tl, j0, j0 + TK, a.sinks)) {
        uint8_t* vt = sm + L::V + s * NB * BLK;
        // The tile's keys fall into runs: [0, s_any) are first tokens that some
        // row sees, of which [0, s_all) are seen by all; then a gap up to the
        // windows, [w_lo, w_all) seen by some, [w_all, w_hi) by all, [w_hi,
        // w_end) by some, and nothing after.  Runs seen by none are cleared,
        // runs seen by some are searched for infinities and NaN.
        auto in = [&](int j) { return max(0, min(TK, j - j0)); };
        const int s_any = in(min(a.sinks, tl.hi_max)), s_all = in(min(a.sinks, tl.hi_min));
        const int w_lo = max(s_any, in(tl.lo_min)), w_end = max(w_lo, in(tl.hi_max));
        const int w_all = max(w_lo, min(w_end, in(tl.lo_max))), w_hi = max(w_all, min(w_end, in(tl.hi_min)));
        // a run of keys: four keys a step, eight lanes a key
        auto clear = [&](int k0, int k1) {
          for (int key = k0 + (lane >> 3); key < k1; key += 4)
#pragma unroll
            for (int kb = 0; kb < NB; ++kb)
              *reinterpret_cast<uint4*>(vt + kb * BLK + key * 128 + ((lane & 7) << 4)) = make_uint4(0, 0, 0, 0);
        };
        bool odd = false;
        auto search = [&](int k0, int k1) {
#pragma unroll 4
          for (int key = k0 + (lane >> 3); key < k1; key += 4)
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) {
              uint4* p = reinterpret_cast<uint4*>(vt + kb * BLK + key * 128 + ((lane & 7) << 4));
              uint4 v = *p;
              if (nonfinite2<T>(v.x) || nonfinite2<T>(v.y) || nonfinite2<T>(v.z) || nonfinite2<T>(v.w)) {
                uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  if ((w[k] & Elem<T>::kExp) == Elem<T>::kExp) w[k] &= 0xFFFF0000u;
                  if (((w[k] >> 16) & Elem<T>::kExp) == Elem<T>::kExp) w[k] &= 0xFFFFu;
                }
                *p = v;
                odd = true;
              }
            }
        };
        search(s_all, s_any);
        clear(s_any, w_lo);
        search(w_lo, w_all);
        search(w_hi, w_end);
        clear(w_end, TK);
        if (odd) s_poison = 1;
        fence_proxy_async_smem();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_VRDY + s));
    }
    if (!ok) s_err = 1;
  }

  tc_fence_before();
  __syncthreads();
  if (warp == W_MMA) {
    tc_fence_after();
    tmem_dealloc(tbase, 512);
  }
  if (tid == 0 && s_err) record_status(a.status, QWM_ERR_TIMEOUT);
}

// The parts of the groups that were cut, in part order: m = max m_p, l = sum l_p
// 2^(m_p - m), O = sum O_p 2^(m_p - m) / l, with m as powers of two.  A CTA takes 64 rows, a warp 8
// of them; lanes 8 rows x 4 groups of 8 channels, so that reads (a part lies
// [channels / 4][row]) and writes are whole sectors.
constexpr int JR = 64;
template <typename T, int D>
__global__ void __launch_bounds__(256) paged_join(const PagedArgs a) {
  grid_begin();
  const int b = blockIdx.z, hk = blockIdx.y, rt = blockIdx.x / (ROWS / JR);
  const int rtiles = gridDim.x / (ROWS / JR);
  Seq sq;
  load_seq(a, b, sq);
  const int64_t rows = (int64_t)sq.qn * a.G, r0 = (int64_t)rt * ROWS;
  if (r0 >= rows) return;
  const int nrow = (int)min((int64_t)ROWS, rows - r0);
  const int tokA = (int)(r0 / a.G), p0 = sq.kv - sq.qn;
  const uint32_t G = (uint32_t)a.G, remA = (uint32_t)(r0 - (int64_t)tokA * a.G);
  const int tokB = tokA + (int)((remA + (uint32_t)nrow - 1) / G);
  const Tiles tl = make_tiles<TK>(p0 + tokA, p0 + tokB, sq.kv, a.block, a.window, a.sinks);
  const int per = max((tl.n + a.nsplit - 1) / a.nsplit, a.min_tiles);
  const int parts = max(1, (tl.n + per - 1) / per);
  const int lane = threadIdx.x & 31;
  const int r = (blockIdx.x % (ROWS / JR)) * JR + (threadIdx.x >> 5) * 8 + (lane & 7);
  if (parts == 1 || r >= nrow) return;
  const int64_t group = ((int64_t)b * a.Hk + hk) * rtiles + rt;
  const float2* ml = a.part_ml + group * a.nsplit * ROWS + r;
  const float4* po = reinterpret_cast<const float4*>(a.part_o) + group * a.nsplit * ROWS * (D / 4) + r;
  constexpr int CB = D / 32, PU = 4;                  // channel blocks of a lane, parts in flight
  float m = -INFINITY, l = 0.0f;
  float4 v[CB][2];
#pragma unroll
  for (int k = 0; k < CB; ++k) v[k][0] = v[k][1] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int pb = 0; pb < parts; pb += PU) {
    float2 w[PU];
    float4 x[PU][CB][2];
#pragma unroll
    for (int u = 0; u < PU; ++u) {
      const int p = min(pb + u, parts - 1);
      w[u] = __ldcg(ml + p * ROWS);
      if (pb + u >= parts) w[u] = make_float2(-INFINITY, 0.0f);
#pragma unroll
      for (int k = 0; k < CB; ++k) {
        const float4* src = po + ((int64_t)p * (D / 4) + 2 * (4 * k + (lane >> 3))) * ROWS;
        x[u][k][0] = __ldcg(src);
        x[u][k][1] = __ldcg(src + ROWS);
      }
    }
    float mn = m;
#pragma unroll
    for (int u = 0; u < PU; ++u) mn = fmaxf(mn, w[u].x);
    const float ref = mn == -INFINITY ? 0.0f : mn;
    const float al = ex2f(m - ref);
    m = mn;
    l *= al;
#pragma unroll
    for (int k = 0; k < CB; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        v[k][h].x *= al; v[k][h].y *= al; v[k][h].z *= al; v[k][h].w *= al;
      }
#pragma unroll
    for (int u = 0; u < PU; ++u) {
      if (pb + u >= parts) break;
      const float f = ex2f(w[u].x - ref);
      l = fmaf(w[u].y, f, l);
#pragma unroll
      for (int k = 0; k < CB; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          v[k][h].x = fmaf(x[u][k][h].x, f, v[k][h].x); v[k][h].y = fmaf(x[u][k][h].y, f, v[k][h].y);
          v[k][h].z = fmaf(x[u][k][h].z, f, v[k][h].z); v[k][h].w = fmaf(x[u][k][h].w, f, v[k][h].w);
        }
    }
  }
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  const int tok = tokA + (int)((remA + r) / G), head = hk * a.G + (int)((remA + r) % G);
  T* dst = static_cast<T*>(a.out) + (sq.q0 + tok) * a.o_tok + (int64_t)head * a.o_head + 8 * (lane >> 3);
#pragma unroll
  for (int k = 0; k < CB; ++k)
    *reinterpret_cast<uint4*>(dst + 32 * k) =
        make_uint4(Elem<T>::pack(v[k][0].x * inv, v[k][0].y * inv), Elem<T>::pack(v[k][0].z * inv, v[k][0].w * inv),
                   Elem<T>::pack(v[k][1].x * inv, v[k][1].y * inv), Elem<T>::pack(v[k][1].z * inv, v[k][1].w * inv));
  if (a.lse && lane < 8) a.lse[(int64_t)head * a.N + sq.q0 + tok] = log_sum<T>(m, l);
}

template <typename T, int D>
cudaError_t go(const PagedArgs& a, const CUtensorMap& map, cudaStream_t s) {
  static bool done[64];
  cudaError_t e = allow_smem(paged_chunk<T, D>, Smem<D>::TOTAL, done);
  if (e != cudaSuccess) return e;
  const int64_t rtiles = ((int64_t)a.max_q * a.G + ROWS - 1) / ROWS;
  e = launch_ahead(paged_chunk<T, D>, dim3((unsigned)(rtiles * a.nsplit), a.Hk, a.B), NT, Smem<D>::TOTAL, s, map, a);
  if (e != cudaSuccess || a.nsplit == 1) return e;
  return launch_ahead(paged_join<T, D>, dim3((unsigned)(rtiles * (ROWS / JR)), a.Hk, a.B), 256, 0, s, a);
}

}  // namespace

PagedPlan plan_chunk(int B, int Hk, int64_t rows, int64_t max_visible, int nsm, bool split) {
  PagedPlan p{};
  p.rows = ROWS;
  const int64_t rtiles = (rows + p.rows - 1) / p.rows;
  const int64_t groups = rtiles * B * Hk;
  p.groups = (int)(groups < 1 << 30 ? groups : 1 << 30);   // (as many are not split)
  p.min_tiles = 4;
  p.nsplit = 1;
  const int64_t tiles = (max_visible + TK - 1) / TK + 2;
  if (split) {
    // the split with the least waves x (tiles of a part + a CTA's fixed cost,
    // about 6 tiles' time), 4 more for the join; parts of at least 4 tiles.  Not
    // past 8 waves, where a split evens out the last one only and the parts' fp32
    // sums grow without end (170 to 256 MB in the first calls past it): 2500 Queries
    // x 64 heads over 8192 keys take 502 us split and 457 whole, 3900 x 40 over 16384
    // 854 either way, over 32768 1604 and 1672.
    int64_t best = 0;
    for (int64_t n = 1; n <= 64 && n * p.min_tiles <= tiles + p.min_tiles - 1; ++n) {
      if (n > 1 && p.groups * n > 8 * (int64_t)nsm) break;
      const int64_t waves = ((int64_t)p.groups * n + nsm - 1) / nsm, cost = waves * ((tiles + n - 1) / n + 6) + (n > 1 ? 4 : 0);
      if (n == 1 || cost < best) {
        best = cost;
        p.nsplit = (int)n;
      }
    }
  }
  return p;
}

cudaError_t launch_paged_chunk(const PagedArgs& a, const CUtensorMap& map, int D, int dtype, cudaStream_t s) {
  if (dtype == QWM_F16) return D == 64 ? go<__half, 64>(a, map, s) : go<__half, 128>(a, map, s);
  return D == 64 ? go<__nv_bfloat16, 64>(a, map, s) : go<__nv_bfloat16, 128>(a, map, s);
}

}  // namespace qwm
