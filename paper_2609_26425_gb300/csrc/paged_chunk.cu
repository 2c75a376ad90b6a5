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
//
// 8-bit pages: the producers bring codes, and a fourth warpgroup makes binary16 tiles of
// them, the Values' guard in one.  What was found on the way (4680 Queries x 40 heads over 34320
// keys; 880 x 12 over 14080): codes through registers, a tile ahead, by three warps of the twelve
// 9465 and 288 us, their loads waited for one after the other; a warpgroup of its own, with
// registers shared out by role, 2643 and 93; codes by TMA 2476 and 95: shared memory then
// is the MMAs' bound, who read 192 KB a tile pair of 128 channels while 64 KB are written.  So
// at 128 channels two CTAs share their MMAs (cta_group::2, M = 256): each makes and holds half of
// a tile's Keys, and half of the Values' channels, and reads 128 KB where 32 KB are written: 2432 and
// 84 (less than the gain a tile, 3.5 K to 3.2 K cycles, for 400 pairs are 5.3 waves of 76);
// with only the last wave cut along the keys 2330, with the registers shared out anew 2260.
// What is left is the chain S, softmax, P V: without softmax and rebuilding the MMAs take 1690
// us (100% of a library product's rate), without exponentials 2200, without rebuilding 2190.
// S in halves of 64 keys, each made while the other half is worked on, reads the Queries twice
// and lost what it won (2500).  At 64 channels a CTA works alone, as with 16-bit pages.
#include <type_traits>

#include "paged.cuh"

namespace qwm {
namespace {
using namespace ptx;

constexpr int TK = 128;
constexpr int ST = 2;                     // K tiles and V tiles in flight
constexpr int BLK = 16384;                // 128 rows x 128 bytes
// 8-bit pages: tiles of K codes, and of V codes, in flight (4680 Queries x 40 heads: two 2287 us,
// three 2254, four 2260)
constexpr int kCodeStages = 3;

enum { B_KFULL = 0, B_KEMPTY = 2, B_VFULL = 4, B_VRDY = 6, B_VEMPTY = 8, B_SFULL = 10, B_QRDY = 12, B_PV = 14,
       B_PFULL = 16 /* tile, half */, B_OFIN = 20,
       B_KREL = 22, B_VREL = 24 /* the second CTA's K and V, to be told to the first */,
       B_CFULL = 26 /* codes: K, V, stage */, B_CEMPTY = B_CFULL + 2 * kCodeStages, N_BAR = B_CEMPTY + 2 * kCodeStages };

constexpr int NQ = 2, ROWS = 128 * NQ;               // row tiles and rows of a CTA
constexpr int W_MMA = 4 * NQ, W_K = W_MMA + 1, W_V = W_MMA + 2;  // W_MMA + 3: the guard
constexpr int W_CODES = W_MMA + 4;                   // 8-bit pages: 4 warps for K and V
constexpr int NT = (4 * NQ + 4) * 32;
// 8-bit pages: a fourth warpgroup makes K and V from codes, and the warps share out the
// registers (65536 in all): softmax, the MMAs' and the producers' warpgroup, the codes'.
constexpr int kRebuild = 4, NT8 = NT + 128;
constexpr int kRegLaunch = 65536 / NT8, kRegSoftmax = 176, kRegMma = 64, kRegCodes = 96;
static_assert(NT8 == 512 && NQ * kRegSoftmax + kRegMma + kRegCodes <= 4 * kRegLaunch, "what the launch has");

template <int D, bool C8>
struct Smem {
  // 8-bit pages of 128 channels: a pair of CTAs shares its MMAs, and each has half of
  // the keys of a K tile and half of the channels of a V tile
  static constexpr bool PAIR = C8 && D == 128;
  static constexpr int GR = PAIR ? 2 * ROWS : ROWS;  // rows of a group (a CTA's, or a pair's)
  static constexpr int NB = D / 64;                  // 64-channel blocks of a tile
  static constexpr int KROWS = PAIR ? TK / 2 : TK, KBLK = KROWS * 128, KST = NB * KBLK;   // of a CTA: keys, bytes
  static constexpr int VCH = PAIR ? D / 2 : D, VST = VCH / 64 * BLK;                      // channels, bytes
  static constexpr int Q = 0;                        // tile i, block k at (i * NB + k) * BLK
  static constexpr int K = NQ * NB * BLK;            // stage s, block k at s * KST + k * KBLK
  static constexpr int V = K + ST * KST;
  // 8-bit pages: tiles of codes [K, V][stage], and their scales [K, V][stage][TK]
  static constexpr int CS = C8 ? kCodeStages : 0, CT = TK * VCH;
  static_assert(KROWS * D == CT, "K and V codes of a CTA");
  static constexpr int CODES = V + ST * VST;
  static constexpr int SCALES = CODES + 2 * CS * CT;
  static constexpr int BAR = SCALES + 2 * CS * TK * 2;
  static constexpr int TOTAL = BAR + N_BAR * 8 + 1024;
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
// P of a new maximum is 2^-kBias, and may grow until 64 of them sum up to kMost before the
// maximum moves.  8-bit pages: binary16 keeps all bits of P down to 2^-16 of the maximum of a
// row's first tile, and none below 2^-27.  Less room to grow costs time: 2^11 (then 2^-19)
// 86 and 2288 us where 2^14 takes 83 and 2276, 2^9 95 and 2317, 2^7 103 and 2395 (880 Queries x
// 12 heads; 4680 x 40).
template <typename T, bool C8>
struct Range {
  static constexpr int kBias = Elem<T>::kBias;
  static constexpr float kMost = pow2(Elem<T>::kTau - kBias);
};
template <typename T>
struct Range<T, true> {
  static constexpr int kBias = -2;
  static constexpr float kMost = 65504.0f;
};
// Natural-log sum-exp of a row: `m` is the power that its P were taken against, l
// their sum.  -inf (and log 0) where nothing was seen, NaN with a NaN sum.
template <int BIAS>
__device__ __forceinline__ float log_sum(float m, float l) {
  return (m - (float)BIAS + log2f(l * pow2(BIAS))) * 0.69314718055994531f;
}

// A warpgroup's registers a thread from here on: fewer than at the launch, or more, for which
// it waits until others have given theirs.
template <int N>
__device__ __forceinline__ void set_registers() {
  static_assert(N % 8 == 0 && N >= 24 && N <= 256, "");
  if constexpr (N < kRegLaunch) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
  else asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}

// K and V of 8-bit pages: warp `w` of four turns a quarter of the CTA's share of each
// tile from codes into binary16, where the TMA of 16-bit pages would have put it, so that
// the MMAs are the same: 16 codes a lane.  Values that no row sees are cleared on the way,
// those that some see and others do not searched (the guard's work; true in *odd where
// something was taken out).  `done` hands a stage of K or V on.  False: a wait ran out.
template <int D, class Done>
__device__ __forceinline__ bool rebuild_tiles(const PagedArgs& a, uint8_t* sm, const Tiles& tl, int t0, int n, int w,
                                              bool* odd, Done done) {
  using L = Smem<D, true>;
  const int lane = threadIdx.x & 31;
  auto bar = [&](int i) { return smem_u32(sm + L::BAR) + 8u * i; };
  auto wait_all = [&](int i, uint32_t ph) -> bool { return __all_sync(0xFFFFFFFFu, mbar_wait(bar(i), ph, a.wait_ns)); };
  // Tile jt of K (NR keys x NC channels here) or V: from codes to its place in the ring,
  // blocks of 64 channels `stride` bytes apart
  auto rebuild = [&](auto rows_, auto channels_, auto masked, int kv, int jt, uint8_t* tile, int stride) {
    constexpr int NR = rows_, NC = channels_, LPR = NC / 16, RPL = 32 / LPR;   // lanes of a row, rows of a load
    constexpr int LOADS = NR / RPL / kRebuild;
    const int c = lane % LPR, row0 = w * (NR / kRebuild) + lane / LPR;
    const int st = kv * L::CS + jt % L::CS;
    const uint8_t* codes = sm + L::CODES + st * L::CT;
    const uint16_t* scales = reinterpret_cast<const uint16_t*>(sm + L::SCALES) + st * TK;
    uint4 x[LOADS];
    uint32_t s2[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = row0 + i * RPL;
      x[i] = *reinterpret_cast<const uint4*>(codes + row * NC + ((NC == 128 ? c ^ (row & 7) : c ^ ((row >> 1) & 3)) << 4));
      s2[i] = scales[row] * 0x10001u;
    }
    // The codes are given back when they are in registers: with the loads only issued, the next
    // copy now and then was there before them (after the tiles at the mask's edges, where copies
    // are far ahead: 1 call in 50 of 4680 Queries x 40 heads).  So which lane tells depends on a
    // value of every load.  (Given back when the tile was written: 2315 us against 2254.)
    uint32_t all = 0;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) all ^= x[i].x ^ s2[i];
    const int teller = __any_sync(0xFFFFFFFFu, all == 0x5A3C96E1u) ? 1 : 0;
    if (lane == teller) mbar_arrive(bar(B_CEMPTY + st));
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = row0 + i * RPL;
      uint32_t h[8];
      from_codes(x[i].x, h[0], h[1]);
      from_codes(x[i].y, h[2], h[3]);
      from_codes(x[i].z, h[4], h[5]);
      from_codes(x[i].w, h[6], h[7]);
#pragma unroll
      for (int k = 0; k < 8; ++k) h[k] = mul_f16x2(h[k], s2[i]);
      if constexpr (masked) {
        const int j = tile_at(tl, t0 + jt) * TK + row;
        if (!any_sees(tl, j, j + 1, a.sinks)) {
#pragma unroll
          for (int k = 0; k < 8; ++k) h[k] = 0u;
        } else if (!all_see(tl, j, j + 1, a.sinks)) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            if (!nonfinite2<__half>(h[k])) continue;
            if ((h[k] & 0x7C00u) == 0x7C00u) h[k] &= 0xFFFF0000u;
            if ((h[k] & 0x7C000000u) == 0x7C000000u) h[k] &= 0xFFFFu;
            *odd = true;
          }
        }
      }
      const uint4 lo = make_uint4(h[0], h[1], h[2], h[3]), hi = make_uint4(h[4], h[5], h[6], h[7]);
      uint8_t* at = tile + (c >> 2) * stride + row * 128;   // channels 16 c ..: chunks 2 c and 2 c + 1 of 8
      const int k0 = (2 * c) & 7, sw = row & 7;
      // the lanes of the upper channels write their second chunk first: no two of the
      // eight lanes of a row on one bank
      const bool flip = NC == 128 && c >= 4;
      *reinterpret_cast<uint4*>(at + (((k0 + flip) ^ sw) << 4)) = flip ? hi : lo;
      *reinterpret_cast<uint4*>(at + (((k0 + !flip) ^ sw) << 4)) = flip ? lo : hi;
    }
    fence_proxy_async_smem();
    __syncwarp();
  };
  using KRows = std::integral_constant<int, L::KROWS>;
  using VChannels = std::integral_constant<int, L::VCH>;
  using All = std::integral_constant<int, D>;
  using Keys = std::integral_constant<int, TK>;
  for (int jt = 0; jt < n; ++jt) {
    const int s = jt & 1, j0 = tile_at(tl, t0 + jt) * TK, cs = jt % L::CS;
    const uint32_t ph = (jt / L::CS) & 1;
    if (!wait_all(B_CFULL + cs, ph)) return false;
    if (jt >= ST && !wait_all(B_KEMPTY + s, ((jt >> 1) - 1) & 1)) return false;
    rebuild(KRows{}, All{}, std::false_type{}, 0, jt, sm + L::K + s * L::KST, L::KBLK);
    done(0, s);
    if (!wait_all(B_CFULL + L::CS + cs, ph)) return false;
    if (jt >= ST && !wait_all(B_VEMPTY + s, ((jt >> 1) - 1) & 1)) return false;
    uint8_t* tile = sm + L::V + s * L::VST;
    if (all_see(tl, j0, j0 + TK, a.sinks)) rebuild(Keys{}, VChannels{}, std::false_type{}, 1, jt, tile, BLK);
    else rebuild(Keys{}, VChannels{}, std::true_type{}, 1, jt, tile, BLK);
    done(1, s);
  }
  return true;
}

// T: the type of Queries and output; C8: 8-bit pages, whose products are taken in
// binary16 (every code x scale is one).
template <typename T, int D, bool C8>
__global__ void __launch_bounds__(C8 ? NT8 : NT, 1) paged_chunk(const __grid_constant__ CUtensorMap map,
                                                                 const __grid_constant__ CUtensorMap half_map,   // pairs: 64 channels
                                                                 const PagedArgs a) {
  using L = Smem<D, C8>;
  constexpr bool PAIR = L::PAIR;
  using Op = Operand<T, C8>;
  constexpr int NB = L::NB;
  extern __shared__ uint8_t raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  __shared__ uint32_t s_tmem;
  __shared__ int s_err, s_poison;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  auto bar = [&](int i) { return smem_u32(sm + L::BAR) + 8u * i; };
  const uint32_t rank = PAIR ? cluster_rank() : 0;    // 0: the CTA that issues the pair's MMAs
  if (tid == 0) {
    for (int s = 0; s < 2; ++s) {
      // (of a pair: this CTA's warps, and for K and V one arrival for all of the other's)
      mbar_init(bar(B_KFULL + s), C8 ? kRebuild + PAIR : 1);
      mbar_init(bar(B_KEMPTY + s), 1);
      mbar_init(bar(B_VFULL + s), 1);
      mbar_init(bar(B_VRDY + s), C8 ? kRebuild + PAIR : 1);
      mbar_init(bar(B_VEMPTY + s), 1);
      mbar_init(bar(B_SFULL + s), 1);
      mbar_init(bar(B_PV + s), 1);
      mbar_init(bar(B_PFULL + 2 * s), PAIR ? 8 : 4);
      mbar_init(bar(B_PFULL + 2 * s + 1), PAIR ? 8 : 4);
      mbar_init(bar(B_QRDY + s), PAIR ? 8 : 4);
      if constexpr (PAIR) {
        mbar_init(bar(B_KREL + s), kRebuild);
        mbar_init(bar(B_VREL + s), kRebuild);
      }
    }
    if constexpr (C8) {
      for (int s = 0; s < 2 * L::CS; ++s) {
        mbar_init(bar(B_CFULL + s), 1);
        mbar_init(bar(B_CEMPTY + s), kRebuild);
      }
    }
    mbar_init(bar(B_OFIN), 1);
    s_err = 0;
    s_poison = 0;
    fence_mbar_init();
  }
  grid_begin();
  int b = blockIdx.z, hk = blockIdx.y;
  const int gx = PAIR ? blockIdx.x >> 1 : blockIdx.x;
  int rtiles, rt, part, nsplit = a.nsplit;
  int64_t cut;                                          // the group's number among those in parts
  if (C8 && a.whole >= 0) {
    // groups in one line: the first `whole` of them as they are, the others in parts
    rtiles = a.rtiles;
    const int y = gx - a.whole, group = y < 0 ? gx : a.whole + y / nsplit;
    part = y < 0 ? 0 : y % nsplit;
    if (y < 0) nsplit = 1;
    cut = group - a.whole;
    rt = rtiles - 1 - group % rtiles;
    b = group / rtiles / a.Hk;
    hk = group / rtiles % a.Hk;
  } else {
    rtiles = (PAIR ? gridDim.x >> 1 : gridDim.x) / nsplit;
    rt = rtiles - 1 - gx % rtiles;                      // the row tiles with the most keys first
    part = gx / rtiles;
    cut = ((int64_t)b * a.Hk + hk) * rtiles + rt;
  }
  Seq sq;
  if (!load_seq(a, b, sq) && rt == rtiles - 1 && part == 0 && hk == 0 && tid == 0) record_status(a.status, QWM_ERR_INVALID_ARG);
  const int64_t rows = (int64_t)sq.qn * a.G;
  const int64_t r0 = (int64_t)rt * L::GR;
  if (r0 >= rows) return;
  const int nrow = (int)min((int64_t)L::GR, rows - r0);
  const int nqt = nrow > L::GR / 2 ? 2 : 1;
  // row tile i holds the group's rows row_at(i) ..: of a pair, 128 of the first CTA, then of the second
  auto row_at = [&](int i) { return PAIR ? 256 * i + 128 * (int)rank : 128 * i; };
  const int p0 = sq.kv - sq.qn;                       // token of the sequence's first row
  // row r0 + i is new token tokA + (remA + i) / G, grouped head (remA + i) % G
  const int tokA = (int)(r0 / a.G);
  const uint32_t G = (uint32_t)a.G, remA = (uint32_t)(r0 - (int64_t)tokA * a.G);
  const int tokB = tokA + (int)((remA + (uint32_t)nrow - 1) / G);
  const Tiles tl = make_tiles<TK>(p0 + tokA, p0 + tokB, sq.kv, a.block, a.window, a.sinks);
  const int per = nsplit == 1 ? max(tl.n, 1) : max((tl.n + nsplit - 1) / nsplit, a.min_tiles);
  const int parts = max(1, (tl.n + per - 1) / per);
  if (part >= parts) return;
  const int t0 = part * per, n = max(0, min(tl.n, t0 + per) - t0);   // this part's tiles: t0 .. t0 + n - 1

  auto wait_all = [&](int i, uint32_t ph) -> bool {
    return __all_sync(0xFFFFFFFFu, mbar_wait(bar(i), ph, a.wait_ns));
  };
  __syncthreads();                                    // the barriers are set up
  if (warp == W_MMA) {
    if constexpr (PAIR) {
      tmem_alloc2(smem_u32(&s_tmem), 512);
      tmem_relinquish2();
    } else {
      tmem_alloc(smem_u32(&s_tmem), 512);
      tmem_relinquish();
    }
  }
  if constexpr (PAIR) {
    tc_fence_before();
    cluster_arrive();                                 // this CTA's barriers and TMEM are there
  }
  int q_up = 0;                                       // 8-bit pages: this thread's row was taken times 2^q_up
  if (warp < W_MMA && (warp >> 2) < nqt) {
    const int i = warp >> 2;
    // Q_i: each warp its 32 rows, a row's 16-byte chunks over neighbouring lanes, RPK rows a load
    uint8_t* sQ = sm + L::Q + i * NB * BLK;
    constexpr int CH = D / 8, RPK = 32 / CH;
    uint4 v[CH];
    {
      const int rr0 = (warp & 3) * 32 + lane / CH;
      const uint32_t r = remA + row_at(i) + rr0, step_t = RPK / G, step_g = RPK % G;
      uint32_t t = r / G, g = r % G;
#pragma unroll
      for (int k = 0; k < CH; ++k) {
        v[k] = make_uint4(0, 0, 0, 0);
        if (row_at(i) + rr0 + k * RPK < nrow)
          v[k] = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + (sq.q0 + tokA + t) * a.q_tok +
                                                 (hk * a.G + (int)g) * a.q_head + (lane % CH) * 8);
        t += step_t;
        g += step_g;
        if (g >= G) { g -= G; ++t; }
      }
    }
    if constexpr (C8 && Elem<T>::bf16) {
      // A row's power of two: each lane has the maxima of CH rows' chunks; they are halved
      // with a lane's at a time, until lane c of CH has row c's.
      uint32_t top[CH];
#pragma unroll
      for (int k = 0; k < CH; ++k) top[k] = finite_max(v[k]);
#pragma unroll
      for (int s = CH / 2; s > 0; s >>= 1)
#pragma unroll
        for (int k = 0; k < s; ++k) {
          const uint32_t mine = lane & s ? top[k + s] : top[k], other = lane & s ? top[k] : top[k + s];
          top[k] = max(mine, __shfl_xor_sync(0xFFFFFFFFu, other, s));
        }
      const int up = row_power(top[0]);
      q_up = __shfl_sync(0xFFFFFFFFu, up, (lane % RPK) * CH + lane / RPK);   // of the softmax thread's row
#pragma unroll
      for (int k = 0; k < CH; ++k) v[k] = scaled_f16(v[k], __shfl_sync(0xFFFFFFFFu, up, (lane & ~(CH - 1)) + k));
    }
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int rr = (warp & 3) * 32 + k * RPK + lane / CH, c = lane % CH;
      *reinterpret_cast<uint4*>(sQ + (c >> 3) * BLK + rr * 128 + (((c & 7) ^ (rr & 7)) << 4)) = v[k];
    }
    fence_proxy_async_smem();
  }
  // The producers and the guard touch no TMEM: their first copies go out while it is
  // being allocated and the Queries come in.  (All warps waiting for the allocation
  // and the Queries loaded after it: 880 Queries x 12 heads 64.0 us against 62.5;
  // three ragged prompts of 64 channels 79.5 against 80.5.)
  // (Of a pair, who reaches into the other CTA waits for its barriers and TMEM; the others
  // before they meet it again.)
  uint32_t tbase = 0;
  const bool reaches = warp <= W_MMA || (warp == W_MMA + 3 && rank == 1);
  if constexpr (PAIR) {
    if (reaches) {
      cluster_wait();
      tc_fence_after();
      tbase = s_tmem;
    }
  } else if (warp <= W_MMA) {
    tc_fence_before();
    named_bar_sync(1, (W_MMA + 1) * 32);
    tc_fence_after();
    tbase = s_tmem;
  }
  const float sl2 = a.scale * 1.4426950408889634f;

  if (warp < W_MMA) {
    // ------------------------------------------------------------ softmax
    if constexpr (C8) set_registers<kRegSoftmax>();
    const int i = warp >> 2, row = tid & 127;
    if (i < nqt) {
      uint8_t* sQ = sm + L::Q + i * NB * BLK;
      constexpr int CH = D / 8;
      __syncwarp();
      if (lane == 0) {
        if (rank == 0) mbar_arrive(bar(B_QRDY + i));
        else mbar_arrive_cluster(mapa(bar(B_QRDY + i), 0));
      }

      const bool has = row_at(i) + row < nrow;
      const int tok = has ? tokA + (int)((remA + row_at(i) + row) / G) : tokB;
      const int head = hk * a.G + (has ? (int)((remA + row_at(i) + row) % G) : 0);
      const Span sp = has ? row_span(p0 + tok, sq.kv, a.block, a.window) : Span{0, 0};
      const uint32_t lrow = (uint32_t)((warp & 3) * 32) << 16;
      const uint32_t tS = tbase + 128 * i + lrow, tO = tbase + 128 * NQ + D * i + lrow;
      float m_run = has ? -INFINITY : 0.0f, l_run = 0.0f;
      const float sr = C8 && Elem<T>::bf16 ? row_scale(sl2, q_up) : sl2;
      const uint64_t SL = f2pack(sr, sr);
      using P = Range<T, C8>;
      // P = 2^(s sr - power(m_run))
      auto power = [&](float m) { return fmaf(m, sr, (float)P::kBias); };
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
      // What all rows of the warp see: tiles that end at all_hi, and begin at all_lo or end in the first tokens
      int all_lo = has ? sp.lo : 0, all_hi = has ? sp.hi : INT32_MAX;
      bool fresh = true;                                // some row may have no maximum yet
      if constexpr (C8) {
        all_lo = __reduce_max_sync(0xFFFFFFFFu, all_lo);
        all_hi = __reduce_min_sync(0xFFFFFFFFu, all_hi);
      }
      bool ok = true;
      for (int jt = 0; jt < n; ++jt) {
        if (!(ok = wait_all(B_SFULL + i, jt & 1))) break;
        tc_fence_after();
        const int j0 = tile_at(tl, t0 + jt) * TK;
        const bool open = C8 ? j0 + TK <= all_hi && (j0 >= all_lo || j0 + TK <= a.sinks)
                             : __all_sync(0xFFFFFFFFu, !has || (j0 + TK <= sp.hi && (j0 >= sp.lo || j0 + TK <= a.sinks)));
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
        if ((!C8 || fresh) && __any_sync(0xFFFFFFFFu, m_run == -INFINITY)) {
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
          if constexpr (C8) fresh = __any_sync(0xFFFFFFFFu, m_run == -INFINITY);
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
            pk[16 * (blk & 1) + (e >> 1)] = Elem<Op>::pack(x, y);
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
            if (__any_sync(0xFFFFFFFFu, sx + sy > P::kMost)) {
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
            // (P is tensor memory, stored and fenced: the other CTA's arrival has nothing to release)
            if (lane == 0) {
              if (rank == 0) mbar_arrive(bar(B_PFULL + 2 * i + half));
              else mbar_arrive_cluster_relaxed(mapa(bar(B_PFULL + 2 * i + half), 0));
            }
          }
        };
        if (open) pass(std::false_type{});
        else pass(std::true_type{});
        if (!ok) break;
      }
      if (ok && n > 0) ok = wait_all(B_OFIN, 0);
      if (!ok) s_err = 1;
      if constexpr (PAIR) cluster_sync();             // what either CTA took out of the Values is known
      if (ok) {
        tc_fence_after();
        const int64_t pr = (cut * nsplit + part) * L::GR + row_at(i) + row;
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
                const int64_t at = (((page * 2 + 1) * a.Hk + hk) << a.page_log2) + (j & ((1 << a.page_log2) - 1));
                uint32_t s2 = 0;
                if (C8) s2 = *reinterpret_cast<const uint16_t*>(a.scales + at) * 0x10001u;
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                  uint32_t w;
                  if (C8) {
                    uint32_t none;
                    from_codes(*reinterpret_cast<const uint16_t*>(static_cast<const uint8_t*>(a.pages) + at * D + c0 + e), w, none);
                    w = mul_f16x2(w, s2);
                  } else {
                    w = *reinterpret_cast<const uint32_t*>(static_cast<const T*>(a.pages) + at * D + c0 + e);
                  }
                  const float2 f = Elem<Op>::unpack(w);
                  if ((w & Elem<Op>::kExp) == Elem<Op>::kExp) v[e] += f.x;
                  if (((w >> 16) & Elem<Op>::kExp) == Elem<Op>::kExp) v[e + 1] += f.y;
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
            float4* d4 = reinterpret_cast<float4*>(a.part_o) + (cut * nsplit + part) * L::GR * (D / 4) +
                         (int64_t)(c0 / 4) * L::GR + row_at(i) + row;
#pragma unroll
            for (int k = 0; k < 8; ++k) d4[k * L::GR] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
          }
        }
        if (parts == 1) {
          __syncwarp();
#pragma unroll 4
          for (int it = 0; it < CH; ++it) {
            const int idx = it * 32 + lane, rr = (warp & 3) * 32 + idx / CH, c = idx % CH;
            if (row_at(i) + rr >= nrow) continue;
            const uint32_t r = remA + row_at(i) + rr;
            *reinterpret_cast<uint4*>(static_cast<T*>(a.out) + (sq.q0 + tokA + r / G) * a.o_tok +
                                      (int64_t)(hk * a.G + (int)(r % G)) * a.o_head + c * 8) =
                *reinterpret_cast<const uint4*>(sQ + (c >> 3) * BLK + rr * 128 + (((c & 7) ^ (rr & 7)) << 4));
          }
        }
        if (has && parts == 1 && a.lse)
          a.lse[(int64_t)head * a.N + sq.q0 + tok] = log_sum<P::kBias>(power(m_run), l_run);
        if (has && parts > 1) a.part_ml[pr] = make_float2(power(m_run), l_run);
      }
    } else if constexpr (PAIR) {
      cluster_sync();
    }
  } else if (C8 && warp >= W_CODES) {
    // ------------------------------------------------------------ K and V from codes
    if constexpr (C8) {
      set_registers<kRegCodes>();
      bool odd = false;
      auto done = [&](int kv, int s) {
        if (odd) s_poison = 1;
        __syncwarp();
        if (lane == 0) mbar_arrive(bar((rank == 0 ? (kv ? B_VRDY : B_KFULL) : (kv ? B_VREL : B_KREL)) + s));
      };
      if (!rebuild_tiles<D>(a, sm, tl, t0, n, warp - W_CODES, &odd, done)) s_err = 1;
      if constexpr (PAIR) {
        cluster_wait();
        if (odd) st_cluster(mapa(smem_u32(&s_poison), rank ^ 1), 1);
        __syncwarp();
        cluster_sync();
      }
    }
  } else {
    if constexpr (C8) set_registers<kRegMma>();
    if (warp == W_MMA && rank == 0) {
    // ------------------------------------------------------------ MMA issue
    // Order per K/V tile j: P0 V(j) in two halves, S0(j+1), P1 V(j), S1(j+1); S_i(j+1) may
    // overwrite P_i(j) because the MMAs of one thread run in issue order.
    const uint32_t e = elect_one();
    const uint64_t dQ = desc_sw128(smem_u32(sm + L::Q)), dK = desc_sw128(smem_u32(sm + L::K));
    const uint64_t dV = PAIR ? desc_sw128(smem_u32(sm + L::V)) : desc_sw128_mn(smem_u32(sm + L::V), BLK);
    auto off = [](int bytes) { return (uint64_t)(bytes >> 4); };
    constexpr uint32_t idS = idesc_f16(PAIR ? 256 : 128, TK, false, Elem<Op>::bf16);
    constexpr uint32_t idPV = idesc_f16(PAIR ? 256 : 128, D, true, Elem<Op>::bf16);
    auto mma_ss = [&](uint32_t d, uint64_t x, uint64_t y, uint32_t acc) {
      if constexpr (PAIR) umma2_ss_e(d, x, y, idS, acc, e);
      else umma_ss_e(d, x, y, idS, acc, e);
    };
    auto mma_ts = [&](uint32_t d, uint32_t x, uint64_t y, uint32_t acc) {
      if constexpr (PAIR) umma2_ts_e(d, x, y, idPV, acc, e);
      else umma_ts_e(d, x, y, idPV, acc, e);
    };
    auto commit = [&](int i) {
      if constexpr (PAIR) umma2_commit_both_e(bar(i), e);
      else commit_e(bar(i), e);
    };
    auto wait_mma = [&](int i, uint32_t ph) -> bool {
      if constexpr (PAIR) return __all_sync(0xFFFFFFFFu, mbar_wait_cluster(bar(i), ph, a.wait_ns));
      else return wait_all(i, ph);
    };
    bool ok = true;
    auto issue_S = [&](int i, int jt) -> bool {
      const int s = jt & 1;
      if (i == 0 && !wait_mma(B_KFULL + s, (jt >> 1) & 1)) return false;
      if (jt == 0 && !wait_mma(B_QRDY + i, 0)) return false;
      tc_fence_after();
#pragma unroll
      for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
          mma_ss(tbase + 128 * i, dQ + off((i * NB + kb) * BLK + ks * 32), dK + off(s * L::KST + kb * L::KBLK + ks * 32),
                 (kb | ks) != 0);
      commit(B_SFULL + i);
      if (i == nqt - 1) commit(B_KEMPTY + s);
      return true;
    };
    if (n > 0) {
      for (int i = 0; i < nqt && ok; ++i) ok = issue_S(i, 0);
      for (int jt = 0; jt < n && ok; ++jt) {
        const int s = jt & 1;
        if (!(ok = wait_mma(B_VRDY + s, (jt >> 1) & 1))) break;
        for (int i = 0; i < nqt; ++i) {
#pragma unroll
          for (int half = 0; half < 2 && ok; ++half) {
            if (!(ok = wait_mma(B_PFULL + 2 * i + half, jt & 1))) break;
            tc_fence_after();
#pragma unroll
            for (int ks = 4 * half; ks < 4 * half + 4; ++ks)
              mma_ts(tbase + 128 * NQ + D * i, tbase + 128 * i + 8 * ks, dV + off(s * L::VST + ks * 2048), (jt | ks) != 0);
            if (half == 0) commit(B_PV + i);
          }
          if (!ok) break;
          if (i == nqt - 1) commit(B_VEMPTY + s);
          if (jt + 1 < n && !(ok = issue_S(i, jt + 1))) break;
        }
      }
      commit(B_OFIN);
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
    // Of 8-bit pages: a box's codes and its scales, CS tiles of each in flight; a CTA of
    // a pair takes its half of a tile's Keys, or its half of the Values' channels.
    constexpr int STAGES = C8 ? L::CS : ST;
    const int full = C8 ? B_CFULL + kv * L::CS : (kv ? B_VFULL : B_KFULL);
    const int empty = C8 ? B_CEMPTY + kv * L::CS : (kv ? B_VEMPTY : B_KEMPTY);
    const int box_log2 = min(a.page_log2, 6);
    const int k0 = PAIR && !kv ? (int)rank * L::KROWS : 0;   // the CTA's first key of a tile
    const int row_bytes = kv ? L::VCH : D;                   // (of codes)
    const int boxes = (kv ? TK : L::KROWS) >> box_log2;
    const int box = C8 ? lane : lane / NB, blk = C8 ? 0 : lane % NB;
    const bool mine = box < boxes;
    const int32_t* trow = a.table + (int64_t)b * a.table_stride;
    const uint32_t ring = C8 ? smem_u32(sm + L::CODES) + kv * L::CS * L::CT + ((box << box_log2) * row_bytes)
                             : smem_u32(sm + (kv ? L::V : L::K)) + blk * BLK + ((box << box_log2) * 128);   // (KBLK is BLK)
    const uint32_t sring = C8 ? smem_u32(sm + L::SCALES) + kv * L::CS * TK * 2 + ((box << box_log2) * 2) : 0u;
    const uint32_t box_bytes = (C8 ? row_bytes + 2u : 128u) << box_log2;
    auto page_of = [&](int jt, bool& want) -> int {
      const int j0 = tile_at(tl, t0 + jt) * TK + k0 + (box << box_log2);
      want = mine && any_sees(tl, j0, j0 + (1 << box_log2), a.sinks);
      return want ? trow[j0 >> a.page_log2] : 0;
    };
    bool want = false, ok = true;
    int page = n > 0 ? page_of(0, want) : 0;
    int jt = 0;
    for (; jt < n && !a.idle; ++jt) {
      const int s = jt % STAGES;
      bool want_n = false;
      int page_n = 0;
      if (jt + 1 < n) page_n = page_of(jt + 1, want_n);   // its latency runs beside the copies
      if (want && (page < 0 || page >= a.num_pages)) {    // not followed: the first page in its place
        record_status(a.status, QWM_ERR_INVALID_ARG);
        page = 0;
      }
      const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, want)) * box_bytes;
      const int y = (tile_at(tl, t0 + jt) * TK + k0 + (box << box_log2)) & ((1 << a.page_log2) - 1);
      if (jt >= STAGES && !(ok = wait_all(empty + s, (jt / STAGES - 1) & 1))) break;
      if (lane == 0) mbar_arrive_expect_tx(bar(full + s), bytes);
      __syncwarp();
      if (want) {
        const int block = (page * 2 + kv) * a.Hk + hk;
        if (PAIR && kv) tma_load_3d(ring + s * L::CT, &half_map, (int)rank * L::VCH, y, block, bar(full + s));
        else tma_load_3d(ring + s * (C8 ? L::CT : NB * BLK), &map, blk * 64, y, block, bar(full + s));
        if (C8) bulk_g2s(sring + s * TK * 2, a.scales + (((int64_t)block << a.page_log2) + y), 2u << box_log2, bar(full + s));
      }
      __syncwarp();
      page = page_n;
      want = want_n;
    }
    if (!ok) s_err = 1;
    // the last copies land before the CTA can end: the roles that wait for them may
    // have given up on them
    for (int u = max(0, jt - STAGES); u < jt; ++u) mbar_wait(bar(full + u % STAGES), (u / STAGES) & 1, kDrainNs);
    } else if (PAIR && rank == 1) {
      // ------------------------------------------------------------ relays
      // Of the second CTA, W_MMA and the last warp tell the first that a stage of K or V is
      // there: a release over the cluster waits for what the SM has in flight, and the
      // warps that make the stages go on meanwhile.
      const int kv = warp != W_MMA;
      bool ok = true;
      for (int jt = 0; jt < n && ok; ++jt) {
        const int s = jt & 1;
        ok = wait_all((kv ? B_VREL : B_KREL) + s, (jt >> 1) & 1);
        if (ok && lane == 0) mbar_arrive_cluster(mapa(bar((kv ? B_VRDY : B_KFULL) + s), 0));
      }
      if (!ok) s_err = 1;
    } else if (!C8) {
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
    if constexpr (PAIR) {
      __syncwarp();
      if (!reaches) cluster_wait();
      cluster_sync();
    }
  }

  tc_fence_before();
  __syncthreads();
  if constexpr (PAIR) cluster_sync();                 // neither frees the pair's TMEM while the other reads it
  if (warp == W_MMA) {
    tc_fence_after();
    if constexpr (PAIR) tmem_dealloc2(tbase, 512);
    else tmem_dealloc(tbase, 512);
  }
  if (tid == 0 && s_err) record_status(a.status, QWM_ERR_TIMEOUT);
}

// The parts of the groups that were cut, in part order: m = max m_p, l = sum l_p
// 2^(m_p - m), O = sum O_p 2^(m_p - m) / l, with m as powers of two.  A CTA takes 64 rows, a warp 8
// of them; lanes 8 rows x 4 groups of 8 channels, so that reads (a part lies
// [channels / 4][row]) and writes are whole sectors.
constexpr int JR = 64;
template <typename T, int D, int BIAS, int GR>
__global__ void __launch_bounds__(256) paged_join(const PagedArgs a) {
  grid_begin();
  int b = blockIdx.z, hk = blockIdx.y, rt = blockIdx.x / (GR / JR), rtiles = gridDim.x / (GR / JR);
  int64_t group;
  if (a.whole >= 0) {                                 // a line of the groups that were cut
    const int g = a.whole + rt;
    group = rt;
    rtiles = a.rtiles;
    rt = rtiles - 1 - g % rtiles;
    b = g / rtiles / a.Hk;
    hk = g / rtiles % a.Hk;
  } else {
    group = ((int64_t)b * a.Hk + hk) * rtiles + rt;
  }
  Seq sq;
  load_seq(a, b, sq);
  const int64_t rows = (int64_t)sq.qn * a.G, r0 = (int64_t)rt * GR;
  if (r0 >= rows) return;
  const int nrow = (int)min((int64_t)GR, rows - r0);
  const int tokA = (int)(r0 / a.G), p0 = sq.kv - sq.qn;
  const uint32_t G = (uint32_t)a.G, remA = (uint32_t)(r0 - (int64_t)tokA * a.G);
  const int tokB = tokA + (int)((remA + (uint32_t)nrow - 1) / G);
  const Tiles tl = make_tiles<TK>(p0 + tokA, p0 + tokB, sq.kv, a.block, a.window, a.sinks);
  const int per = max((tl.n + a.nsplit - 1) / a.nsplit, a.min_tiles);
  const int parts = max(1, (tl.n + per - 1) / per);
  const int lane = threadIdx.x & 31;
  const int r = (blockIdx.x % (GR / JR)) * JR + (threadIdx.x >> 5) * 8 + (lane & 7);
  if (parts == 1 || r >= nrow) return;
  const float2* ml = a.part_ml + group * a.nsplit * GR + r;
  const float4* po = reinterpret_cast<const float4*>(a.part_o) + group * a.nsplit * GR * (D / 4) + r;
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
      w[u] = __ldcg(ml + p * GR);
      if (pb + u >= parts) w[u] = make_float2(-INFINITY, 0.0f);
#pragma unroll
      for (int k = 0; k < CB; ++k) {
        const float4* src = po + ((int64_t)p * (D / 4) + 2 * (4 * k + (lane >> 3))) * GR;
        x[u][k][0] = __ldcg(src);
        x[u][k][1] = __ldcg(src + GR);
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
  if (a.lse && lane < 8) a.lse[(int64_t)head * a.N + sq.q0 + tok] = log_sum<BIAS>(m, l);
}

template <typename T, int D, bool C8>
cudaError_t go(PagedArgs a, const CUtensorMap& map, const CUtensorMap& half_map, cudaStream_t s) {
  using L = Smem<D, C8>;
  static bool done[64];
  cudaError_t e = allow_smem(paged_chunk<T, D, C8>, L::TOTAL, done);
  if (e != cudaSuccess) return e;
  const int64_t rtiles = ((int64_t)a.max_q * a.G + L::GR - 1) / L::GR, groups = rtiles * a.Hk * a.B;
  const unsigned wide = L::PAIR ? 2 : 1;
  a.rtiles = (int)rtiles;
  dim3 grid((unsigned)(rtiles * a.nsplit * wide), a.Hk, a.B), join((unsigned)(rtiles * (L::GR / JR)), a.Hk, a.B);
  if (a.whole >= 0) {
    grid = dim3((unsigned)((a.whole + (groups - a.whole) * a.nsplit) * wide));
    join = dim3((unsigned)((groups - a.whole) * (L::GR / JR)));
  }
  e = launch_ahead(paged_chunk<T, D, C8>, grid, C8 ? NT8 : NT, L::TOTAL, s, (int)wide, map, half_map, a);
  if (e != cudaSuccess || a.nsplit == 1) return e;
  return launch_ahead(paged_join<T, D, Range<T, C8>::kBias, L::GR>, join, 256, 0, s, 1, a);
}
template <typename T, bool C8>
cudaError_t pick(const PagedArgs& a, const CUtensorMap& map, const CUtensorMap& half_map, int D, cudaStream_t s) {
  return D == 64 ? go<T, 64, C8>(a, map, half_map, s) : go<T, 128, C8>(a, map, half_map, s);
}

}  // namespace

PagedPlan plan_chunk(int B, int Hk, int D, int64_t rows, int64_t max_visible, int nsm, bool split, bool codes) {
  PagedPlan p{};
  const bool pair = codes && D == 128;                                // a group is a pair of CTAs'
  p.rows = pair ? 2 * ROWS : ROWS;
  if (pair) nsm /= 2;
  const int64_t rtiles = (rows + p.rows - 1) / p.rows;
  const int64_t groups = rtiles * B * Hk;
  p.groups = (int)(groups < 1 << 30 ? groups : 1 << 30);   // (as many are not split)
  p.min_tiles = 4;
  p.nsplit = 1;
  p.whole = -1;
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
  // Of 8-bit pages also: full waves of whole groups, and only what would be a part of a
  // wave cut (4680 Queries x 40 heads, 400 pairs in 5.3 waves: 2330 us against 2432).
  const int64_t full = p.groups / nsm * nsm, tail = p.groups - full;
  if (split && codes && p.groups < 1 << 28 && full > 0 && tail > 0) {
    int64_t best = (int64_t)((p.groups * (int64_t)p.nsplit + nsm - 1) / nsm) * ((tiles + p.nsplit - 1) / p.nsplit + 6) +
                   (p.nsplit > 1 ? 4 : 0);
    for (int64_t n = 2; n <= 64 && n * p.min_tiles <= tiles + p.min_tiles - 1; ++n) {
      const int64_t cost = full / nsm * (tiles + 6) + (tail * n + nsm - 1) / nsm * ((tiles + n - 1) / n + 6) + 4;
      if (cost < best) {
        best = cost;
        p.nsplit = (int)n;
        p.whole = (int)full;
      }
    }
  }
  return p;
}

cudaError_t launch_paged_chunk(const PagedArgs& a, const CUtensorMap& map, const CUtensorMap& half_map, int D, int dtype,
                               cudaStream_t s) {
  if (a.scales)
    return dtype == QWM_F16 ? pick<__half, true>(a, map, half_map, D, s) : pick<__nv_bfloat16, true>(a, map, half_map, D, s);
  return dtype == QWM_F16 ? pick<__half, false>(a, map, half_map, D, s) : pick<__nv_bfloat16, false>(a, map, half_map, D, s);
}

}  // namespace qwm
