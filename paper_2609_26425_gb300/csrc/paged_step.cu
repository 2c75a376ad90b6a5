// paged_step.cu -- attention of a few rows of a sequence over its pages: single
// new tokens and short drafts (Query tokens x grouped heads <= 16 rows; over 8-bit pages up
// to 32, in blocks of 8).
//
// Mathematics: softmax over the visible keys with a running maximum m and sum l
// per row (O and l scaled by 2^((m_old - m_new) c) when m grows), so one pass
// over K and V suffices.  The bound is HBM: K and V of the visible tokens are
// read once per cache head for all the grouped Query heads.
//
// The tiles of all (sequence, cache head) groups form one line, which the CTAs (one
// per SM) share out evenly whatever the lengths are; a CTA walks its stretch
// group by group.  Two producer warps, one of K and one of V, keep a ring of tiles
// (64 or 128 keys) in flight by TMA.  One warp for both sent them one after the
// other: 32 sequences of 100 to 30000 keys x 8 heads, window 8192, took 84.3 us and
// take 80.8 with two; one token over 517 keys x 12 heads in pages of 16, where a
// tile is many copies, 9.9 and 8.1.  Of eight more warps four take a quarter of a
// tile's keys each, the other four those of the next tile, and carry their own
// m, l and O through the group (no barrier between them in the loop); then they
// are merged through shared memory.  The rows are the M = 16 side of mma.sync: a
// tcgen05 tile would be 128 rows high for the 1 to 16 used here, and its TMEM
// round trip is longer than the whole of a short step.  P is rounded to the cache's
// type for the product, after its sum (error against 64 bits 1.0 to 1.1 times the
// fp32 form's).
// A group cut by the ends of stretches is joined by the CTA that finishes last,
// in the order of the keys, so the result does not depend on which one that is.
#include <type_traits>

#include "paged.cuh"

namespace qwm {
namespace {
using namespace ptx;

constexpr int kWarps = 8;                // consumer warps
constexpr int NT = (kWarps + 2) * 32;    // and two producers, of K and of V
// What a group costs a CTA beside its tiles (Queries, merge, output: about 5 K
// cycles, and as much again where 8-bit pages have to be unpacked at the mask's edges),
// in tiles' time (1.3 K cycles when all CTAs stream).  Of 8-bit pages, 32 sequences of 100
// to 30000 keys x 8 heads, window 8192: 52 us with 4, 45.4 with 6, 44.5 with 8, 50.6 with 14
// (tiles of 128 keys; of 256, 21 drafts of 4 tokens over 64 to 20000 keys: 24.3 with 4, 22.4 with 5).
template <bool C8, int KP = 2>
constexpr int group_cost() { return !C8 ? 4 : KP == 4 ? 5 : 8; }

// Of 8-bit pages P enters the products as binary16, 2^15 at a row's maximum: from 2^-29 of
// it on with all its bits, down to 2^-39 at all (with 1 at the maximum from 2^-14 on, which
// the many keys beside a first token that draws most of the weight can lie below).
template <bool C8>
constexpr float kTop = C8 ? 15.0f : 0.0f;

// KP 16-key groups of a warp.  A tile's chain of products, exponentials and
// products takes as long for two groups as for one, so two where the chain bounds
// (64 channels; whole groups), one where HBM does and finer slots keep it busier
// (128 channels on the line: 131071 keys 86 us with one, 91 with two; 517 keys x 12
// whole groups 8.9 and 7.6; all four with one producer warp for K and V).
// Of 8-bit pages two groups as well: a tile is half the bytes, and its chain the same
// (131071 keys 56 us, with one 69); of 64 channels four where groups are long (plan_step).
// N8: at most 8 rows, which are the N side of the products then.
template <int D, int KP_, bool C8, bool N8>
struct Shape {
  static_assert(C8 || !N8, "");
  static constexpr int KP = KP_;
  static constexpr int TK = 64 * KP;                           // keys per tile
  static constexpr int SLOT = TK * D * (C8 ? 1 : 2);           // bytes of a K or V tile
  static constexpr int NS = C8 ? 131072 / SLOT : (SLOT == 32768 ? 4 : 8);   // slots of the ring: K, V, K, V, ...
  static_assert(NS % 4 == 0, "an even number of tiles: a slot belongs to one warp group");
  static constexpr int ROWS = N8 ? 8 : 16;
  static constexpr int MERGE = NS * SLOT;                      // the warps' O [warp][ROWS][D], beside the ring so that
                                                               // the next group's tiles come in meanwhile
  static constexpr int SCALES = MERGE + kWarps * ROWS * D * 4; // 8-bit pages: the tiles' scales [slot][TK]
  // Queries of 9 to 16 rows of 128 channels lie in shared memory as fragments [k16 step][lane]:
  // in registers, others spill (21 drafts of 4 tokens over 64 to 20000 keys 38.9 us, so 36.4)
  static constexpr bool QS = C8 && !N8 && D == 128;
  static constexpr int QUERIES = SCALES + (C8 ? NS * TK * 2 : 0);
  static constexpr int TOTAL = QUERIES + (QS ? (D / 16) * 32 * 16 : 0) + 1024;
};

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

// Byte of 16-byte chunk `chunk` (8 channels) of key `key` in a tile [D / 64][TK
// keys][128 bytes], 128-byte swizzled.
template <int TK>
__device__ __forceinline__ uint32_t at(int key, int chunk) {
  return (uint32_t)((chunk >> 3) * (TK * 128) + key * 128 + (((chunk & 7) ^ (key & 7)) << 4));
}

// The same of a tile of codes [TK keys][D bytes]: 16 channels a chunk, swizzled by 128 or
// 64 bytes.
template <int D>
__device__ __forceinline__ uint32_t at_code(int key, int chunk) {
  return (uint32_t)(key * D + ((D == 128 ? chunk ^ (key & 7) : chunk ^ ((key >> 1) & 3)) << 4));
}

__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {   // a >= 0, b > 0
  return ((a | b) >> 32) ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}

// An 8 x 8 block of 16-bit values over the warp, transposed.
__device__ __forceinline__ uint32_t transpose8(uint32_t w) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(w));
  return r;
}

// Whether scales (binary16, any number in words of one or two) are such that their products with
// every code are binary16 numbers: 0 or a power of two from 2^-14 to 2^7.
struct CodeScales {
  uint32_t all = 0, top = 0;
  __device__ __forceinline__ void add(uint32_t w) {
    all |= w;
    top = vmax_u16x2(top, w);
  }
  __device__ __forceinline__ bool exact() const {
    return (all & 0x83FF83FFu) == 0u && (top & 0xFFFFu) <= 0x5800u && (top >> 16) <= 0x5800u;
  }
};

// Codes enter the products as binary16: a lane's word of four of a Key's channels is its
// fragment of one k16 step (the channels of a step in the order 4 tq .. 4 tq + 3 for Q and
// K alike), a transposed word of Values two tokens' pairs of channels, which are put in
// order before the conversion.  The Keys' scales multiply the logits where code x scale is a binary16 number
// for every code, and the fragments where one may not be (a scale that a caller wrote, or one at
// the ends of the range): every kernel rounds code x scale to binary16.  The Values' multiply the
// fragments (P times a scale would leave binary16's range).  Up to 8 rows (N8) are the
// N = 8 side, keys and channels M = 16 (S^T = K Q^T, O^T += V^T P^T): a conversion then feeds
// half as many MMAs and no half of a fragment is idle rows (131071 keys, 8 rows: 56 us
// against 59 with the rows as M; 32 sequences, 5 rows: 44.5 against 48; 9 to 12 rows in two
// such blocks took 28.6 us where rows as M take 26).  More warps lost: 12 59 us, 16 76.
template <typename T, int D, int KP, bool C8, bool N8>
__global__ void __launch_bounds__(NT, 1) paged_step(const __grid_constant__ CUtensorMap map, const PagedArgs a) {
  using L = Shape<D, KP, C8, N8>;
  using Op = Operand<T, C8>;
  constexpr int NS = L::NS, TK = L::TK, ROWS = L::ROWS, kGroupCost = group_cost<C8, KP>();
  constexpr int KS = D / 16;                       // k16 steps of Q K^T, n16 blocks of P V
  extern __shared__ uint8_t raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  __shared__ uint64_t bars[2 * NS];
  __shared__ float s_ml[kWarps][ROWS][2];
  __shared__ int64_t s_scan[kWarps + 2], s_first;
  __shared__ Seq s_sq;
  __shared__ Tiles s_tl;
  __shared__ int s_last, s_seq;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // tiles of a group of sequence b (one for a group that has rows and sees
  // nothing: its output is written all the same)
  auto tiles_of = [&](int b, Seq& sq, Tiles& tl) -> int {
    // on the line CTA 0 looks at every sequence, of whole groups each CTA at its own
    if (!load_seq(a, b, sq) && (a.nsplit == 1 || blockIdx.x == 0)) record_status(a.status, QWM_ERR_INVALID_ARG);
    if (sq.qn == 0) return 0;
    tl = make_tiles<TK>(sq.kv - sq.qn, sq.kv - 1, sq.kv, a.block, a.window, a.sinks);
    return max(tl.n, 1);
  };
  // a sequence's groups: a cache head's rows, or blocks of 8 of them, side by side
  auto blocks_of = [&](const Seq& of) -> int { return N8 && a.blocks > 1 ? (of.qn * a.G + 7) / 8 : 1; };
  auto groups_of = [&](const Seq& of) -> int { return a.Hk * blocks_of(of); };
  auto full = [&](int s) { return smem_u32(&bars[s]); };
  auto empty = [&](int s) { return smem_u32(&bars[NS + s]); };
  if (tid == 0) {
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      mbar_init(full(s), C8 ? 33 : 1);               // (the producer's, and of 8-bit pages each lane's scales)
      mbar_init(empty(s), kWarps / 2);
    }
    fence_mbar_init();
  }
  grid_begin();
  // The line: a group of sequence b takes n(b) + kGroupCost places, its tiles
  // last; sequence b's groups follow those of the sequences before it.  A scan
  // over the sequences gives the total and the sequence in which this CTA's
  // stretch begins: up to 32 sequences by each warp for itself, more by the CTA,
  // each thread with a run of sequences.  Without a workspace, a CTA takes the
  // group of its number.
  const bool split = a.nsplit > 1;
  Seq sq;
  Tiles tl;
  int b, n, hk;                                    // hk: group of the sequence
  int64_t x0, x1, g0, share = 0;
  if (split) {
    const bool alone = a.B <= 32;
    const int who = alone ? lane : tid, run = alone ? 1 : (a.B + NT - 1) / NT;
    const int b0 = min(a.B, who * run), b1 = min(a.B, b0 + run);
    int64_t mine = 0;
    for (int i = b0; i < b1; ++i) {
      n = tiles_of(i, sq, tl);
      mine += n ? (int64_t)(n + kGroupCost) * groups_of(sq) : 0;
    }
    int64_t incl = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t x = __shfl_up_sync(0xFFFFFFFFu, incl, d);
      if (lane >= d) incl += x;
    }
    int64_t before = incl - mine, total = __shfl_sync(0xFFFFFFFFu, incl, 31);
    if (!alone) {
      if (lane == 31) s_scan[warp] = incl;
      __syncthreads();
      total = 0;
#pragma unroll
      for (int w = 0; w < kWarps + 2; ++w) {
        if (w < warp) before += s_scan[w];
        total += s_scan[w];
      }
    }
    share = max(divide(total + gridDim.x - 1, gridDim.x), (int64_t)a.min_tiles);
    x0 = blockIdx.x * share;
    if (x0 >= total) return;
    x1 = min(total, x0 + share);
    const bool here = x0 >= before && x0 < before + mine;
    if (alone) {
      // lane `src` has the sequence
      const int src = __ffs(__ballot_sync(0xFFFFFFFFu, here)) - 1;
      auto from = [&](auto v) { return __shfl_sync(0xFFFFFFFFu, v, src); };
      b = src;
      sq.q0 = from(sq.q0);
      sq.qn = from(sq.qn);
      sq.kv = from(sq.kv);
      tl.lo_min = from(tl.lo_min);
      tl.lo_max = from(tl.lo_max);
      tl.hi_min = from(tl.hi_min);
      tl.hi_max = from(tl.hi_max);
      tl.n_win = from(tl.n_win);
      tl.w_start = from(tl.w_start);
      tl.n = from(tl.n);
      g0 = from(before);
      __syncthreads();                              // the barriers are set up
    } else {
      if (here) {
        int64_t at = before;
        for (int i = b0; i < b1; ++i) {
          n = tiles_of(i, sq, tl);
          const int64_t len = n ? (int64_t)(n + kGroupCost) * groups_of(sq) : 0;
          if (x0 < at + len) {
            s_seq = i;
            s_first = at;
            s_sq = sq;
            s_tl = tl;
            break;
          }
          at += len;
        }
      }
      __syncthreads();
      b = s_seq;
      sq = s_sq;
      tl = s_tl;
      g0 = s_first;
    }
    n = max(tl.n, 1);
    hk = (int)divide(x0 - g0, n + kGroupCost);
    g0 += (int64_t)hk * (n + kGroupCost);
  } else {
    b = blockIdx.x / (a.Hk * a.blocks);
    hk = blockIdx.x % (a.Hk * a.blocks);
    n = tiles_of(b, sq, tl);
    if (n == 0 || hk >= groups_of(sq)) return;
    x0 = g0 = 0;
    x1 = n + kGroupCost;
    __syncthreads();
  }
  // The CTA's piece of the current group: tiles t0 .. t1 - 1, none if t0 >= t1.
  int t0, t1;
  auto piece = [&]() {
    const int64_t first = g0 + kGroupCost;
    t0 = (int)max((int64_t)0, x0 - first);
    t1 = (int)min((int64_t)n, x1 - first);
  };
  auto next_group = [&]() -> bool {
    g0 += n + kGroupCost;
    if (g0 >= x1) return false;
    if (++hk == groups_of(sq)) {
      hk = 0;
      do n = tiles_of(++b, sq, tl); while (n == 0);
    }
    return true;
  };

  if (warp >= kWarps) {
    // ---------------------------------------------------------- producers of K and V
    // lane = box * 2 + channel half (of codes: box); a box is the part of a page (at most 64
    // tokens of it) that lies in the tile.  Boxes that no row sees are not read.  The table
    // is read for as many tiles at once as there are lanes for their boxes, while those
    // before are sent: with a lookup for each tile its latency set the pace of short tiles.
    const int kv = warp - kWarps;
    const int box_log2 = min(a.page_log2, 6), boxes = TK >> box_log2, per = 32 / boxes;
    const int box = C8 ? lane : lane >> 1, half = C8 ? 0 : lane & 1;
    const bool mine = box < boxes && half * 64 < D;
    const uint32_t dst = smem_u32(sm) + (C8 ? (box << box_log2) * D : half * (TK * 128) + ((box << box_log2) * 128));
    const uint32_t box_bytes = (C8 ? D : 128u) << box_log2;
    const int skey = 8 * lane, sbox = skey >> box_log2;   // scales: eight keys a lane, 16 bytes
    bool ok = true;
    int i = 0;                                     // tiles sent
    do {
      piece();
      t1 = min(t1, tl.n);
      const int32_t* trow = a.table + (int64_t)b * a.table_stride;
      const int head = hk / blocks_of(sq);
      // this lane's entry: box lane % boxes of tile t + lane / boxes
      auto ask = [&](int t, bool& want) -> int {
        t += lane / boxes;
        const int j0 = tile_at(tl, t) * TK + ((lane % boxes) << box_log2);
        want = t < t1 && any_sees(tl, j0, j0 + (1 << box_log2), a.sinks);
        return want ? trow[j0 >> a.page_log2] : 0;
      };
      bool wants = false, wants_n = false;
      int pages = 0, pages_n = t0 < t1 ? ask(t0, wants_n) : 0, at = per;
      for (int t = t0; t < t1 && !a.idle; ++t, ++at) {
        if (at == per) {
          at = 0;
          wants = wants_n;
          pages = pages_n;
          pages_n = ask(t + per, wants_n);
          if (wants && (pages < 0 || pages >= a.num_pages)) {   // not followed: the first page in its place
            record_status(a.status, QWM_ERR_INVALID_ARG);
            pages = 0;
          }
        }
        const int src = at * boxes + box;          // (< 32 where mine)
        const int page = __shfl_sync(0xFFFFFFFFu, pages, src & 31);
        const bool want = __shfl_sync(0xFFFFFFFFu, (int)wants, src & 31) && mine;
        const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, want)) * box_bytes;
        const int y = (tile_at(tl, t) * TK + (box << box_log2)) & ((1 << a.page_log2) - 1);
        const int s = (2 * i + kv) % NS;
        if (i >= NS / 2 && !(ok = __all_sync(0xFFFFFFFFu, mbar_wait(empty(s), (i / (NS / 2) - 1) & 1, a.wait_ns)))) break;
        if (lane == 0) mbar_arrive_expect_tx(full(s), bytes);
        __syncwarp();
        if (want) {
          const int block = (page * 2 + kv) * a.Hk + head;
          tma_load_3d(dst + s * L::SLOT, &map, half * 64, y, block, full(s));
        }
        if constexpr (C8) {
          // A copy of its own for each box's scales costs as much as its codes: 131071 keys in
          // pages of 16 tokens 62.6 us, so 55.9; 517 keys x 12 heads 7.9 and 7.5; in pages of 64 with 64
          // channels 37.0 and 38.0.
          const int spage = __shfl_sync(0xFFFFFFFFu, pages, (at * boxes + sbox) & 31);
          const bool swant = __shfl_sync(0xFFFFFFFFu, (int)wants, (at * boxes + sbox) & 31) && skey < TK;
          if (swant)
            cp_async16(smem_u32(sm) + L::SCALES + s * (TK * 2) + 2 * skey,
                       a.scales + ((((int64_t)spage * 2 + kv) * a.Hk + head) << a.page_log2) +
                           ((tile_at(tl, t) * TK + skey) & ((1 << a.page_log2) - 1)));
          cp_async_arrive(full(s));
        }
        __syncwarp();
        ++i;
      }
    } while (ok && next_group());
    if (!ok && lane == 0) record_status(a.status, QWM_ERR_TIMEOUT);
    // The last copies land before this warp ends, and so before the CTA can: the
    // consumers may have given up on them.  Otherwise this is the wait the
    // consumers are in as well.
    for (int u = max(0, i - NS / 2); u < i; ++u) mbar_wait(full((2 * u + kv) % NS), (u / (NS / 2)) & 1, kDrainNs);
    return;
  }

  // ------------------------------------------------------------ consumers
  const float sl2 = a.scale * 1.4426950408889634f;
  // The maxima that warps and CTAs hand on are in units of q k^T; with 8-bit pages the powers that P was taken
  // against, since a row's q k^T may be past fp32 there where its logits are not (bf16 Queries have a scale
  // for each row).
  const float unit = C8 ? 1.0f : sl2;
  const int g = lane >> 2, tq = lane & 3;
  const int wg = warp >> 2, key0 = (warp & 3) * 16 * KP;                // tile parity, first key of the tile
  const int mrow = lane & 7, mi = lane >> 3;
  const int kkey = key0 + (mi >> 1) * 8 + mrow, kch = mi & 1;           // K: (keys 0-7 | 8-15) x (chunk, chunk + 1)
  const int vkey = key0 + (mi & 1) * 8 + mrow, vch = mi >> 1;           // V (and codes): the same, keys innermost
  const int maxrows = a.blocks > 1 ? 8 : a.max_q * a.G;
  float* so = reinterpret_cast<float*>(sm + L::MERGE);                  // [warp][ROWS][D]
  bool ok = true;                                                       // no wait of this warp has run out
  int filled = 0;                                                       // slots of the pieces before
  // A slot of Values goes back when they are in registers.  An arrival waits neither for loads that
  // are under way nor for the products that use them (the chunk kernel lost a stage of codes to
  // the next copy that way), so which lane tells depends on a sum that each load of the tile has gone into:
  // `sum(nb)` of every block that a load covers.  (Of Keys the vote on the maximum does that.)
  auto give_back = [&](int slot, auto sum) {
    uint32_t all = 0;
#pragma unroll
    for (int nb = 0; nb < KS; nb += C8 ? 2 : 1) all ^= __float_as_uint(sum(nb));
    const int teller = __any_sync(0xFFFFFFFFu, all == 0x5A3C96E1u) ? 1 : 0;
    if (lane == teller) mbar_arrive(empty(slot));
  };
  do {
    piece();
    if (t0 >= t1) continue;
    const int nb = blocks_of(sq), head = hk / nb, r0 = N8 ? 8 * (hk - head * nb) : 0;
    const int rows = N8 ? min(sq.qn * a.G - r0, 8) : sq.qn * a.G;       // <= ROWS, of the head's from r0 on
    const int t_end = min(t1, tl.n);
    const int64_t group = (int64_t)b * (a.Hk * a.blocks) + hk, first = g0 + kGroupCost;
    const bool whole = first >= x0 && first + n <= x1;                  // the group is this CTA's alone
    const int64_t c0 = whole ? 0 : divide(first, share), c1 = whole ? 0 : divide(first + n - 1, share);   // its CTAs
    const int parts = (int)(c1 - c0) + 1;
    const int p0 = sq.kv - sq.qn;
    if constexpr (N8) {
      // S^T and O^T: this lane has rows 2 tq + x (index x), of keys g and g + 8 and of
      // channels 2 g and 2 g + 1 of 16
      float o[KS][4], m_run[2], l_run[2], slr[2];
      uint32_t qf[KS][2];
      int hi[2], lo[2];
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[k][e] = 0.0f;
      {
        // Queries as B: this lane row g's channels 4 tq .. of each k16 step
        const bool has = g < rows;
        const int tok = has ? (r0 + g) / a.G : 0;
        const T* src = static_cast<const T*>(a.q) + (sq.q0 + tok) * a.q_tok + (int64_t)(head * a.G + (has ? (r0 + g) % a.G : 0)) * a.q_head;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const uint2 w = has ? *reinterpret_cast<const uint2*>(src + ks * 16 + tq * 4) : make_uint2(0u, 0u);
          qf[ks][0] = w.x;
          qf[ks][1] = w.y;
        }
        int up = 0;
        if constexpr (Elem<T>::bf16) {
          uint32_t top = 0;
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) top = max(top, finite_max(make_uint4(qf[ks][0], qf[ks][1], 0u, 0u)));
          top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
          top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
          up = row_power(top);
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            qf[ks][0] = scaled_f16(qf[ks][0], up);
            qf[ks][1] = scaled_f16(qf[ks][1], up);
          }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int r = 2 * tq + x;
          m_run[x] = -INFINITY;
          l_run[x] = 0.0f;
          slr[x] = sl2;
          if constexpr (Elem<T>::bf16) slr[x] = row_scale(sl2, __shfl_sync(0xFFFFFFFFu, up, 4 * r));
          const Span sp = r < rows ? row_span(p0 + (r0 + r) / a.G, sq.kv, a.block, a.window) : Span{0, 0};
          hi[x] = sp.hi;
          lo[x] = sp.lo;
        }
      }
      // (this warp group's tiles: as below)
      for (int t = t0 + (((filled >> 1) + wg) & 1); t < t_end && ok; t += 2) {
        const int i = filled + 2 * (t - t0), s = i % NS;                   // slots s and s + 1
        const int j0 = tile_at(tl, t) * TK + key0;                         // this warp's keys: j0 .. j0 + 16 KP - 1
        if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(full(s), (i / NS) & 1, a.wait_ns)))) break;
        const uint32_t kb = smem_u32(sm) + s * L::SLOT, vb = kb + L::SLOT;
        const uint8_t* sc_k = sm + L::SCALES + s * (TK * 2) + 2 * key0;
        const uint8_t* sc_v = sc_k + TK * 2;
        const bool open = all_see(tl, j0, j0 + 16 * KP, a.sinks), any = any_sees(tl, j0, j0 + 16 * KP, a.sinks);
        uint32_t pf[KP][2];
        if (any) {
          float sc[KP][2][4];                          // two sums each: half the chain of MMAs
#pragma unroll
          for (int kp = 0; kp < KP; ++kp)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[kp][0][e] = sc[kp][1][e] = 0.0f;
          uint32_t hs[KP][2];                          // scales of keys g and g + 8
          CodeScales kind;
#pragma unroll
          for (int kp = 0; kp < KP; ++kp)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              hs[kp][x] = *reinterpret_cast<const uint16_t*>(sc_k + 2 * (kp * 16 + 8 * x + g));
              kind.add(hs[kp][x]);
            }
          const bool exact = __all_sync(0xFFFFFFFFu, kind.exact());
          auto products = [&](auto scaled) {
#pragma unroll
            for (int ks = 0; ks < KS; ks += 2)
#pragma unroll
              for (int kp = 0; kp < KP; ++kp) {
                uint32_t w[4];                         // (keys 0-7 | 8-15) x (step ks, ks + 1)
                ldsm4(kb + at_code<D>(vkey + 16 * kp, ks + vch), w);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                  uint32_t af[4];
                  from_codes(w[2 * x], af[0], af[2]);
                  from_codes(w[2 * x + 1], af[1], af[3]);
                  if constexpr (scaled) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) af[e] = mul_f16x2(af[e], hs[kp][e & 1] * 0x10001u);
                  }
                  Elem<Op>::mma(sc[kp][x], af, qf[ks + x][0], qf[ks + x][1]);
                }
              }
          };
          if (exact) products(std::false_type{});
          else products(std::true_type{});
          bool grow = false;
          float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
          for (int kp = 0; kp < KP; ++kp) {
            const float f0 = exact ? Elem<__half>::unpack(hs[kp][0]).x : 1.0f, f1 = exact ? Elem<__half>::unpack(hs[kp][1]).x : 1.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float& v = sc[kp][0][e];
              v = (v + sc[kp][1][e]) * (e < 2 ? f0 : f1);
              if (!open && !sees(j0 + kp * 16 + g + (e < 2 ? 0 : 8), lo[e & 1], hi[e & 1], a.sinks)) v = -INFINITY;
              top[e & 1] = fmaxf(top[e & 1], v);
            }
          }
          // running maximum of each row, moved only when a key of this slice is above it: the
          // eight lanes of a row agree through three shuffles then
          grow = top[0] > m_run[0] || top[1] > m_run[1];
          if (__any_sync(0xFFFFFFFFu, grow)) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              float v = top[x];
              v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 4));
              v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 8));
              v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 16));
              const float mn = fmaxf(m_run[x], v);
              const float al = mn == m_run[x] ? 1.0f : ex2f((m_run[x] - mn) * slr[x]);
              m_run[x] = mn;
              l_run[x] *= al;
#pragma unroll
              for (int k = 0; k < KS; ++k) {
                o[k][x] *= al;
                o[k][2 + x] *= al;
              }
            }
          }
          // a row that has seen nothing yet keeps 0 as its reference: 2^-inf = 0
          const float mb[2] = {m_run[0] == -INFINITY ? 0.0f : fmaf(m_run[0], slr[0], -kTop<C8>),
                               m_run[1] == -INFINITY ? 0.0f : fmaf(m_run[1], slr[1], -kTop<C8>)};
#pragma unroll
          for (int kp = 0; kp < KP; ++kp) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = ex2f(fmaf(sc[kp][0][e], slr[e & 1], -mb[e & 1]));
            l_run[0] += v[0] + v[2];
            l_run[1] += v[1] + v[3];
            pf[kp][0] = transpose8(Elem<Op>::pack(v[0], v[1]));   // to B: row g, keys 2 tq and 2 tq + 1
            pf[kp][1] = transpose8(Elem<Op>::pack(v[2], v[3]));
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(s));
        if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(full(s + 1), (i / NS) & 1, a.wait_ns)))) break;
        // Values as A, times their scales: channels 2 g and 2 g + 1 of 16 (blocks nb and nb + 1),
        // keys 2 tq, 2 tq + 1 and those plus 8
        auto values = [&](int kp, int nb, uint32_t (&af)[2][4]) {
          uint32_t w[4];                               // (keys 0-7 | 8-15) x (16 channels, the next 16)
          ldsm4t(vb + at_code<D>(vkey + 16 * kp, nb + vch), w);
          const uint32_t s0 = *reinterpret_cast<const uint32_t*>(sc_v + 2 * (kp * 16 + tq * 2));
          const uint32_t s1 = *reinterpret_cast<const uint32_t*>(sc_v + 2 * (kp * 16 + 8 + tq * 2));
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            uint32_t even, odd;
            from_codes(__byte_perm(w[x], 0, 0x3120), even, odd);
            af[x >> 1][2 * (x & 1)] = mul_f16x2(even, x & 1 ? s1 : s0);
            af[x >> 1][2 * (x & 1) + 1] = mul_f16x2(odd, x & 1 ? s1 : s0);
          }
        };
        if (open) {
#pragma unroll
          for (int kp = 0; kp < KP; ++kp)
#pragma unroll
            for (int nb = 0; nb < KS; nb += 2) {
              uint32_t af[2][4];
              values(kp, nb, af);
#pragma unroll
              for (int x = 0; x < 2; ++x) Elem<Op>::mma(o[nb + x], af[x], pf[kp][0], pf[kp][1]);
            }
        } else if (any) {
          // as below: what no row sees is cleared, what some see and others do not is taken
          // token by token where it is not finite
          auto keep = [&](int klo, int khi, int j) -> uint32_t {
            return (sees(j, klo, khi, a.sinks) ? 0xFFFFu : 0u) | (sees(j + 1, klo, khi, a.sinks) ? 0xFFFF0000u : 0u);
          };
#pragma unroll 1
          for (int kp = 0; kp < KP; ++kp) {
            const int ja = j0 + kp * 16 + tq * 2;
            const uint32_t ma = keep(tl.lo_min, tl.hi_max, ja), mb = keep(tl.lo_min, tl.hi_max, ja + 8);
            uint32_t b0 = pf[0][0], b1 = pf[0][1];
#pragma unroll
            for (int k = 1; k < KP; ++k)
              if (kp == k) {
                b0 = pf[k][0];
                b1 = pf[k][1];
              }
            bool odd = false;
            if (sq.qn > 1) {
#pragma unroll 1
              for (int nb = 0; nb < KS; nb += 2) {
                uint32_t af[2][4];
                values(kp, nb, af);
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                  for (int e = 0; e < 4; ++e) odd |= nonfinite2<Op>(af[x][e] & (e < 2 ? ma : mb));
              }
              odd = __any_sync(0xFFFFFFFFu, odd);
            }
            const int turns = odd ? sq.qn : 1;
            for (int tk = 0; tk < turns; ++tk) {
              uint32_t wa = ma, wb = mb;
              if (odd) {
                const Span sp = row_span(p0 + tk, sq.kv, a.block, a.window);
                wa = keep(sp.lo, sp.hi, ja);
                wb = keep(sp.lo, sp.hi, ja + 8);
              }
              const bool own[2] = {!odd || (r0 + 2 * tq) / a.G == tk, !odd || (r0 + 2 * tq + 1) / a.G == tk};
#pragma unroll
              for (int nb = 0; nb < KS; nb += 2) {
                uint32_t af[2][4];
                values(kp, nb, af);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                  af[x][0] &= wa; af[x][1] &= wa; af[x][2] &= wb; af[x][3] &= wb;
                  float acc[4];
#pragma unroll
                  for (int e = 0; e < 4; ++e) acc[e] = o[nb + x][e];
                  Elem<Op>::mma(acc, af[x], b0, b1);
#pragma unroll
                  for (int e = 0; e < 4; ++e)
                    if (own[e & 1]) o[nb + x][e] = acc[e];
                }
              }
            }
          }
        }
        give_back(s + 1, [&](int nb) { return o[nb][0]; });
      }
      filled += 2 * max(0, t_end - t0);
      if (!ok && lane == 0) record_status(a.status, QWM_ERR_TIMEOUT);

      // -------------------------------------------------------- the warps' (max, sum, O) of the piece
      named_bar_sync(1, kWarps * 32);                  // the last piece's have been read
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = 2 * tq + x;
        float l = l_run[x];                            // the eight lanes of a row hold its sum in parts
        l += __shfl_xor_sync(0xFFFFFFFFu, l, 4);
        l += __shfl_xor_sync(0xFFFFFFFFu, l, 8);
        l += __shfl_xor_sync(0xFFFFFFFFu, l, 16);
        if (r >= rows) continue;
        if (g == 0) {
          s_ml[warp][r][0] = fmaf(m_run[x], slr[x], -kTop<C8>);   // what P is taken against
          s_ml[warp][r][1] = l;
        }
#pragma unroll
        for (int k = 0; k < KS; ++k)
          *reinterpret_cast<float2*>(so + ((warp * ROWS + r) * D + k * 16 + g * 2)) =
              make_float2(o[k][x], o[k][2 + x]);
      }
    } else {
      // the fragments of mma.sync: this lane has rows g and g + 8 (index rr)
      float o[2 * KS][4];
      float m_run[2], l_run[2];
      uint32_t qf[KS][4];
      float slr[2] = {sl2, sl2};                                          // scale of a row's logits, as powers of two
      int hi[2], lo[2];
#pragma unroll
      for (int k = 0; k < 2 * KS; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[k][e] = 0.0f;
#pragma unroll
      for (int rr = 0; rr < 2; ++rr) {
        m_run[rr] = -INFINITY;
        l_run[rr] = 0.0f;
        const int r = rr * 8 + g;
        const bool has = r < rows;
        const int tok = has ? r / a.G : 0;
        const Span sp = has ? row_span(p0 + tok, sq.kv, a.block, a.window) : Span{0, 0};
        hi[rr] = sp.hi;
        lo[rr] = sp.lo;
        const T* src = static_cast<const T*>(a.q) + (sq.q0 + tok) * a.q_tok + (int64_t)(head * a.G + (has ? r % a.G : 0)) * a.q_head;
        if constexpr (C8) {
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            const uint2 w = has ? *reinterpret_cast<const uint2*>(src + ks * 16 + tq * 4) : make_uint2(0u, 0u);
            qf[ks][rr] = w.x;
            qf[ks][2 + rr] = w.y;
          }
        } else {
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            qf[ks][rr] = has ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + tq * 2) : 0u;
            qf[ks][2 + rr] = has ? *reinterpret_cast<const uint32_t*>(src + ks * 16 + 8 + tq * 2) : 0u;
          }
        }
      }
      if constexpr (C8 && Elem<T>::bf16) {
        // (after all loads: its branch for infinities would hold up each of them; the drafts above
        // 36.4 us, so 31.0)
#pragma unroll
        for (int rr = 0; rr < 2; ++rr) {
          uint32_t top = 0;
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) top = max(top, finite_max(make_uint4(qf[ks][rr], qf[ks][2 + rr], 0u, 0u)));
          top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
          top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
          const int up = row_power(top);
#pragma unroll
          for (int ks = 0; ks < KS; ++ks) {
            qf[ks][rr] = scaled_f16(qf[ks][rr], up);
            qf[ks][2 + rr] = scaled_f16(qf[ks][2 + rr], up);
          }
          slr[rr] = row_scale(sl2, up);
        }
      }
      uint4* qs = reinterpret_cast<uint4*>(sm + L::QUERIES) + lane;
      if constexpr (L::QS) {
        // each warp writes all of them, the same values (nobody reads the last piece's any more)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qs[32 * ks] = make_uint4(qf[ks][0], qf[ks][1], qf[ks][2], qf[ks][3]);
        __syncwarp();
      }
      // This warp group's tiles are those of its parity in the CTA's count of tiles,
      // so that a slot of the ring is always the same group's: a group that did not
      // wait for every use of a slot could take the phase before the one it waits
      // for as done (a parity tells only two apart).
      for (int t = t0 + (((filled >> 1) + wg) & 1); t < t_end && ok; t += 2) {
        const int i = filled + 2 * (t - t0), s = i % NS;                   // slots s and s + 1
        const int j0 = tile_at(tl, t) * TK + key0;                         // this warp's keys: j0 .. j0 + 16 KP - 1
        if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(full(s), (i / NS) & 1, a.wait_ns)))) break;
        const uint32_t kb = smem_u32(sm) + s * L::SLOT, vb = kb + L::SLOT;
        const bool open = all_see(tl, j0, j0 + 16 * KP, a.sinks), any = any_sees(tl, j0, j0 + 16 * KP, a.sinks);
        uint32_t pf[KP][4];
        // scales of this lane's keys (2 tq, 2 tq + 1) of eight, as binary16
        auto scales_at = [&](int slot, int key) -> uint32_t {
          return *reinterpret_cast<const uint32_t*>(sm + L::SCALES + slot * (TK * 2) + 2 * (key0 + key + tq * 2));
        };
        // B fragments of P V for the channels of two n8 blocks, times their scales
        auto values = [&](int kp, int nb, uint32_t (&bf)[4]) { ldsm4t(vb + at<TK>(vkey + 16 * kp, 2 * nb + vch), bf); };
        // of four n8 blocks (nb even): block 2 nb has the even channels of 16, 2 nb + 1 the odd ones
        auto code_values = [&](int kp, int nb, uint32_t (&bf)[2][4]) {
          uint32_t w[4];                               // (keys 0-7 | 8-15) x (16 channels, the next 16)
          ldsm4t(vb + at_code<D>(vkey + 16 * kp, nb + vch), w);
          const uint32_t s0 = scales_at(s + 1, kp * 16), s1 = scales_at(s + 1, kp * 16 + 8);
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            uint32_t even, odd;
            from_codes(__byte_perm(w[x], 0, 0x3120), even, odd);
            bf[x >> 1][x & 1] = mul_f16x2(even, x & 1 ? s1 : s0);
            bf[x >> 1][2 + (x & 1)] = mul_f16x2(odd, x & 1 ? s1 : s0);
          }
        };
        if (any) {
          float sc[KP][2][4];
#pragma unroll
          for (int kp = 0; kp < KP; ++kp)
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int e = 0; e < 4; ++e) sc[kp][k][e] = 0.0f;
          if constexpr (C8) {
            CodeScales kind;
#pragma unroll
            for (int kp = 0; kp < KP; ++kp)
#pragma unroll
              for (int k = 0; k < 2; ++k) kind.add(scales_at(s, kp * 16 + k * 8));
            const bool exact = __all_sync(0xFFFFFFFFu, kind.exact());
            auto products = [&](auto scaled) {
#pragma unroll
              for (int ks = 0; ks < KS; ks += 2) {
                uint32_t qa[2][4];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                  if constexpr (L::QS) {
                    const uint4 v = qs[32 * (ks + x)];
                    qa[x][0] = v.x; qa[x][1] = v.y; qa[x][2] = v.z; qa[x][3] = v.w;
                  } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) qa[x][e] = qf[ks + x][e];
                  }
                }
#pragma unroll
                for (int kp = 0; kp < KP; ++kp) {
                  uint32_t w[4];                       // (keys 0-7 | 8-15) x (step ks, ks + 1)
                  ldsm4(kb + at_code<D>(vkey + 16 * kp, ks + vch), w);
#pragma unroll
                  for (int x = 0; x < 4; ++x) {
                    uint32_t b0, b1;
                    from_codes(w[x], b0, b1);
                    if constexpr (scaled) {            // (this lane's key is g of eight here)
                      const uint32_t s2 = *reinterpret_cast<const uint16_t*>(sm + L::SCALES + s * (TK * 2) +
                                                                             2 * (key0 + kp * 16 + (x & 1) * 8 + g)) * 0x10001u;
                      b0 = mul_f16x2(b0, s2);
                      b1 = mul_f16x2(b1, s2);
                    }
                    Elem<Op>::mma(sc[kp][x & 1], qa[x >> 1], b0, b1);
                  }
                }
              }
            };
            if (exact) {
              products(std::false_type{});
#pragma unroll
              for (int kp = 0; kp < KP; ++kp)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  const float2 f = Elem<Op>::unpack(scales_at(s, kp * 16 + k * 8));
#pragma unroll
                  for (int e = 0; e < 4; ++e) sc[kp][k][e] *= e & 1 ? f.y : f.x;
                }
            } else {
              products(std::true_type{});
            }
          } else {
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
              for (int kp = 0; kp < KP; ++kp) {
                uint32_t bf[4];
                ldsm4(kb + at<TK>(kkey + 16 * kp, 2 * ks + kch), bf);
                Elem<Op>::mma(sc[kp][0], qf[ks], bf[0], bf[1]);
                Elem<Op>::mma(sc[kp][1], qf[ks], bf[2], bf[3]);
              }
          }
          if (!open) {
#pragma unroll
            for (int kp = 0; kp < KP; ++kp)
#pragma unroll
              for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (!sees(j0 + kp * 16 + k * 8 + tq * 2 + (e & 1), lo[e >> 1], hi[e >> 1], a.sinks)) sc[kp][k][e] = -INFINITY;
          }
          // running maximum of each row, moved only when a key of this slice is
          // above it: the four lanes of a row agree through two shuffles then
          bool grow = false;
          float top[2];
#pragma unroll
          for (int rr = 0; rr < 2; ++rr) {
            top[rr] = -INFINITY;
#pragma unroll
            for (int kp = 0; kp < KP; ++kp)
              top[rr] = fmaxf(top[rr], fmaxf(fmaxf(sc[kp][0][2 * rr], sc[kp][0][2 * rr + 1]),
                                             fmaxf(sc[kp][1][2 * rr], sc[kp][1][2 * rr + 1])));
            grow |= top[rr] > m_run[rr];
          }
          if (__any_sync(0xFFFFFFFFu, grow)) {
#pragma unroll
            for (int rr = 0; rr < 2; ++rr) {
              float v = top[rr];
              v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 1));
              v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 2));
              const float mn = fmaxf(m_run[rr], v);
              const float al = mn == m_run[rr] ? 1.0f : ex2f((m_run[rr] - mn) * slr[rr]);
              m_run[rr] = mn;
              l_run[rr] *= al;
#pragma unroll
              for (int k = 0; k < 2 * KS; ++k) {
                o[k][2 * rr] *= al;
                o[k][2 * rr + 1] *= al;
              }
            }
          }
          // a row that has seen nothing yet keeps 0 as its reference: 2^-inf = 0
          const float mb0 = m_run[0] == -INFINITY ? 0.0f : fmaf(m_run[0], slr[0], -kTop<C8>);
          const float mb1 = m_run[1] == -INFINITY ? 0.0f : fmaf(m_run[1], slr[1], -kTop<C8>);
#pragma unroll
          for (int kp = 0; kp < KP; ++kp)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const float v0 = ex2f(fmaf(sc[kp][k][0], slr[0], -mb0)), v1 = ex2f(fmaf(sc[kp][k][1], slr[0], -mb0));
              const float w0 = ex2f(fmaf(sc[kp][k][2], slr[1], -mb1)), w1 = ex2f(fmaf(sc[kp][k][3], slr[1], -mb1));
              l_run[0] += v0 + v1;
              l_run[1] += w0 + w1;
              pf[kp][2 * k] = Elem<Op>::pack(v0, v1);
              pf[kp][2 * k + 1] = Elem<Op>::pack(w0, w1);
            }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(s));
        if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(full(s + 1), (i / NS) & 1, a.wait_ns)))) break;
        if (open) {
#pragma unroll
          for (int kp = 0; kp < KP; ++kp)
#pragma unroll
            for (int nb = 0; nb < KS; nb += C8 ? 2 : 1) {
              uint32_t bf[2][4];
              if constexpr (C8) code_values(kp, nb, bf);
              else values(kp, nb, bf[0]);
#pragma unroll
              for (int x = 0; x < (C8 ? 2 : 1); ++x) {
                Elem<Op>::mma(o[2 * (nb + x)], pf[kp], bf[x][0], bf[x][1]);
                Elem<Op>::mma(o[2 * (nb + x) + 1], pf[kp], bf[x][2], bf[x][3]);
              }
            }
        } else if (any) {
          // Keys that no row sees may hold anything (0 x inf is not 0): their
          // Values are cleared in the fragments.  Keys that some rows see and
          // others do not (drafts of several tokens): if one holds an infinity
          // or a NaN, the product is taken token by token and only that
          // token's rows keep it.
          auto keep = [&](int klo, int khi, int j) -> uint32_t {
            return (sees(j, klo, khi, a.sinks) ? 0xFFFFu : 0u) | (sees(j + 1, klo, khi, a.sinks) ? 0xFFFF0000u : 0u);
          };
          constexpr int kTurns = C8 ? 1 : KP;          // (unrolled, 8-bit pages spill)
#pragma unroll kTurns
          for (int kp = 0; kp < KP; ++kp) {
            uint32_t pr[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              pr[e] = pf[0][e];
#pragma unroll
              for (int k = 1; k < KP; ++k)
                if (kp == k) pr[e] = pf[k][e];
            }
            const int ja = j0 + kp * 16 + tq * 2;
            const uint32_t ma = keep(tl.lo_min, tl.hi_max, ja), mb = keep(tl.lo_min, tl.hi_max, ja + 8);
            bool odd = false;
            if (sq.qn > 1) {
#pragma unroll
              for (int nb = 0; nb < KS; nb += C8 ? 2 : 1) {
                uint32_t bf[2][4];
                if constexpr (C8) code_values(kp, nb, bf);
                else values(kp, nb, bf[0]);
#pragma unroll
                for (int x = 0; x < (C8 ? 2 : 1); ++x)
                  odd |= nonfinite2<Op>(bf[x][0] & ma) || nonfinite2<Op>(bf[x][1] & mb) || nonfinite2<Op>(bf[x][2] & ma) ||
                         nonfinite2<Op>(bf[x][3] & mb);
              }
              odd = __any_sync(0xFFFFFFFFu, odd);
            }
            const int turns = odd ? sq.qn : 1;
            for (int tk = 0; tk < turns; ++tk) {
              uint32_t wa = ma, wb = mb;
              bool own[2];
#pragma unroll
              for (int rr = 0; rr < 2; ++rr) own[rr] = !odd || (rr * 8 + g) / a.G == tk;
              if (odd) {
                const Span sp = row_span(p0 + tk, sq.kv, a.block, a.window);
                wa = keep(sp.lo, sp.hi, ja);
                wb = keep(sp.lo, sp.hi, ja + 8);
              }
#pragma unroll
              for (int nb = 0; nb < KS; nb += C8 ? 2 : 1) {
                uint32_t bf[2][4];
                if constexpr (C8) code_values(kp, nb, bf);
                else values(kp, nb, bf[0]);
#pragma unroll
                for (int k = 0; k < (C8 ? 4 : 2); ++k) {
                  float acc[4];
#pragma unroll
                  for (int e = 0; e < 4; ++e) acc[e] = o[2 * nb + k][e];
                  Elem<Op>::mma(acc, pr, bf[k >> 1][2 * (k & 1)] & wa, bf[k >> 1][2 * (k & 1) + 1] & wb);
#pragma unroll
                  for (int e = 0; e < 4; ++e)
                    if (own[e >> 1]) o[2 * nb + k][e] = acc[e];
                }
              }
            }
          }
        }
        give_back(s + 1, [&](int nb) { return o[2 * nb][0]; });
      }
      filled += 2 * max(0, t_end - t0);
      if (!ok && lane == 0) record_status(a.status, QWM_ERR_TIMEOUT);

      // -------------------------------------------------------- the warps' (max, sum, O) of the piece
      named_bar_sync(1, kWarps * 32);                  // the last piece's have been read
#pragma unroll
      for (int rr = 0; rr < 2; ++rr) {
        const int r = rr * 8 + g;
        float l = l_run[rr];                           // the four lanes of a row hold its sum in parts
        l += __shfl_xor_sync(0xFFFFFFFFu, l, 1);
        l += __shfl_xor_sync(0xFFFFFFFFu, l, 2);
        if (r >= rows) continue;
        if (tq == 0) {
          s_ml[warp][r][0] = C8 ? fmaf(m_run[rr], slr[rr], -kTop<C8>) : m_run[rr];
          s_ml[warp][r][1] = l;
        }
        if constexpr (C8) {
#pragma unroll
          for (int k = 0; k < 2 * KS; k += 2)
            *reinterpret_cast<float4*>(so + ((warp * ROWS + r) * D + k * 8 + tq * 4)) =
                make_float4(o[k][2 * rr], o[k + 1][2 * rr], o[k][2 * rr + 1], o[k + 1][2 * rr + 1]);
        } else {
#pragma unroll
          for (int k = 0; k < 2 * KS; ++k)
            *reinterpret_cast<float2*>(so + ((warp * ROWS + r) * D + k * 8 + tq * 2)) = make_float2(o[k][2 * rr], o[k][2 * rr + 1]);
        }
      }
    }
    named_bar_sync(1, kWarps * 32);
    auto emit = [&](int r, int c, float m, float l, float4 v) {
      const int tok = (r0 + r) / a.G, h = head * a.G + (r0 + r) % a.G;
      const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
      T* dst = static_cast<T*>(a.out) + (sq.q0 + tok) * a.o_tok + (int64_t)h * a.o_head + 4 * c;
      *reinterpret_cast<uint2*>(dst) = make_uint2(Elem<T>::pack(v.x * inv, v.y * inv), Elem<T>::pack(v.z * inv, v.w * inv));
      if (a.lse && c == 0) a.lse[(int64_t)h * a.N + sq.q0 + tok] = m * (C8 ? 0.69314718055994531f : a.scale) + logf(l);   // -inf + log 0; NaN with a NaN l
    };
    // (m, l, O) of row r's channels 4c .. over the first `count` entries of s_ml and so
    auto merge = [&](int count, int r, int c, float& m, float& l, float4& v) {
      m = -INFINITY;
      for (int w = 0; w < count; ++w) m = fmaxf(m, s_ml[w][r][0]);
      const float ref = m == -INFINITY ? 0.0f : m;
      l = 0.0f;
      v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int w = 0; w < count; ++w) {
        const float f = ex2f((s_ml[w][r][0] - ref) * unit);
        const float4 x = *reinterpret_cast<const float4*>(so + ((w * ROWS + r) * D + 4 * c));
        l = fmaf(s_ml[w][r][1], f, l);
        v.x = fmaf(x.x, f, v.x); v.y = fmaf(x.y, f, v.y); v.z = fmaf(x.z, f, v.z); v.w = fmaf(x.w, f, v.w);
      }
    };
    for (int idx = tid; idx < rows * (D / 4); idx += kWarps * 32) {
      const int r = idx / (D / 4), c = idx % (D / 4);
      float m, l;
      float4 v;
      merge(kWarps, r, c, m, l, v);
      if (parts == 1) {
        emit(r, c, m, l, v);
      } else {
        // a CTA's places: 0 for a group that began before its stretch, 1 for one that begins in it
        const int64_t pr = (2 * (int64_t)blockIdx.x + (first >= x0 ? 1 : 0)) * maxrows + r;
        *reinterpret_cast<float4*>(a.part_o + pr * D + 4 * c) = v;
        if (c == 0) a.part_ml[pr] = make_float2(m, l);
      }
    }
    if (parts == 1) continue;
    // -------------------------------------------------------- the CTA that arrives last joins all parts
    __threadfence();
    named_bar_sync(1, kWarps * 32);
    if (tid == 0) s_last = atomicAdd(a.counter + group, 1) == parts - 1;
    named_bar_sync(1, kWarps * 32);
    if (!s_last) continue;
    __threadfence();
    // part p's rows: the first CTA's second place, the others' first
    auto place = [&](int p) { return (2 * (c0 + p) + (p == 0 ? 1 : 0)) * maxrows; };
    // A warp takes whole rows (where there are fewer rows than warps and more
    // parts than a warp has in flight, the warps share a row's parts out), a lane
    // four channels.  Of 8-bit pages the warps always share: one trip to memory for
    // ten parts (16384 keys x 8 heads, joins of 19 parts: 16.8 us a call with 20 parts in flight
    // and one warp a row, 14.9).
    constexpr int LPR = D / 4, RPW = 32 / LPR;        // lanes per row, rows per warp at a time
    constexpr int PU = C8 ? 10 : 20;                  // parts in flight
    const int rr = (rows + RPW - 1) / RPW;
    const int slices = rr > 4 || parts <= (C8 ? 2 : PU) ? 1 : (rr > 2 ? 2 : (rr > 1 ? 4 : 8)), sl = warp % slices;
    const int q0 = parts * sl / slices, q1 = parts * (sl + 1) / slices;
    for (int rb = (warp / slices) * RPW; rb < rows; rb += (kWarps / slices) * RPW) {
      const int r = rb + lane / LPR, c = lane % LPR;
      float m = -INFINITY, l = 0.0f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r >= rows) continue;
      for (int p = q0; p < q1; p += PU) {
        float2 ml[PU];
        float4 x[PU];
#pragma unroll
        for (int u = 0; u < PU; ++u) {
          const int64_t at_p = place(min(p + u, q1 - 1)) + r;
          ml[u] = __ldcg(&a.part_ml[at_p]);
          x[u] = __ldcg(reinterpret_cast<const float4*>(a.part_o + at_p * D + 4 * c));
        }
        float mn = m;
#pragma unroll
        for (int u = 0; u < PU; ++u) mn = fmaxf(mn, ml[u].x);
        const float ref = mn == -INFINITY ? 0.0f : mn;
        const float al = ex2f((m - ref) * unit);
        m = mn;
        l *= al;
        v.x *= al; v.y *= al; v.z *= al; v.w *= al;
#pragma unroll
        for (int u = 0; u < PU; ++u) {
          if (p + u >= q1) break;
          const float f = ex2f((ml[u].x - ref) * unit);
          l = fmaf(ml[u].y, f, l);
          v.x = fmaf(x[u].x, f, v.x); v.y = fmaf(x[u].y, f, v.y); v.z = fmaf(x[u].z, f, v.z); v.w = fmaf(x[u].w, f, v.w);
        }
      }
      if (slices == 1) {
        emit(r, c, m, l, v);
      } else {
        *reinterpret_cast<float4*>(so + ((sl * ROWS + r) * D + 4 * c)) = v;
        if (c == 0) {
          s_ml[sl][r][0] = m;
          s_ml[sl][r][1] = l;
        }
      }
    }
    if (slices > 1) {
      named_bar_sync(1, kWarps * 32);
      for (int idx = tid; idx < rows * (D / 4); idx += kWarps * 32) {
        const int r = idx / (D / 4), c = idx % (D / 4);
        float m, l;
        float4 v;
        merge(slices, r, c, m, l, v);
        emit(r, c, m, l, v);
      }
    }
    if (tid == 0) a.counter[group] = 0;
  } while (next_group());
}

template <typename T, int D, int KP, bool C8, bool N8>
cudaError_t go(const PagedArgs& a, const CUtensorMap& map, cudaStream_t s) {
  constexpr int smem = Shape<D, KP, C8, N8>::TOTAL;
  static bool done[64];
  cudaError_t e = allow_smem(paged_step<T, D, KP, C8, N8>, smem, done);
  if (e != cudaSuccess) return e;
  return launch_ahead(paged_step<T, D, KP, C8, N8>, dim3((unsigned)(a.nsplit > 1 ? a.nsplit : a.B * a.Hk * a.blocks)), NT, smem, s, 1,
                      map, a);
}
template <typename T, int D>
cudaError_t pick(const PagedArgs& a, const CUtensorMap& map, cudaStream_t s) {
  if (a.scales) {
    const bool few = a.blocks > 1 || (int64_t)a.max_q * a.G <= 8;
    if constexpr (D == 64)
      if (a.wide) return few ? go<T, D, 4, true, true>(a, map, s) : go<T, D, 4, true, false>(a, map, s);
    return few ? go<T, D, 2, true, true>(a, map, s) : go<T, D, 2, true, false>(a, map, s);
  }
  if constexpr (D == 128)
    if (a.nsplit > 1) return go<T, D, 1, false, false>(a, map, s);
  return go<T, D, 2, false, false>(a, map, s);
}

}  // namespace

// Blocks that a cache head's rows are taken in, each a group of its own that reads the head's
// keys again (from L2 while it holds them): 1: all at once, 0: not by this kernel.  In us, codes, by the SMs' and
// the groups' number: of 128 channels 16 rows at once (as M) and in two blocks: 4 heads x 600 keys
// 10.9 and 8.6, x 40000 33.1 and 23.3, 64 heads x 2000 19.6 and 16.0, 32 x 8000 25.0 and 28.5, 256 x 600 22.1
// and 33.4.  20 rows by the chunk kernel and in three blocks: 4 x 600 17.9 and 9.0, 4 x 40000 49.9 and
// 27.6, 256 x 600 71.7 and 46.0; 32 rows in four 18.3 and 9.1, 50.1 and 31.8, 73.7 and 58.7.  Codes past
// L2 change nothing in that, since the chunk kernel's chain is as far from HBM: 64 x 40000 437 and 294 (20 rows), 386
// (32); 256 x 8000 (530 MB) 358 and 243, 322; 128 x 40000 791 and 572, 759; 256 x 40000 (2.6 GB) 1500 and 1505 (32 rows).  Of 64
// channels 9 to 16 rows lose in blocks; 24 rows by the chunk kernel and in three: 4 x 600 12.5 and
// 7.9, 32 x 40000 105 and 90, 64 x 600 13.4 and 14.9; 32 rows in four: 4 x 40000 36.3 and 23.3, 32 x
// 8000 30.9 and 33.1.
int step_blocks(int B, int Hk, int D, int64_t rows, int64_t max_visible, int nsm, bool codes) {
  if (!codes || rows <= 8) return rows <= kStepRows ? 1 : 0;
  const int64_t blocks = (rows + 7) / 8, groups = (int64_t)B * Hk, keys = groups * max_visible;
  if (blocks > 4) return 0;
  const bool wave = groups * blocks <= nsm;                           // a CTA for each block at once
  if (rows <= kStepRows) return D == 128 && wave && keys <= 200000 ? (int)blocks : 1;
  return D == 128 || (wave && (blocks <= 3 || keys <= 200000)) ? (int)blocks : 0;
}

PagedPlan plan_step(int B, int Hk, int D, int rows, int64_t max_visible, int nsm, bool split, bool codes) {
  PagedPlan p{};
  p.step = 1;
  p.blocks = step_blocks(B, Hk, D, rows, max_visible, nsm, codes);
  p.groups = B * Hk * p.blocks;
  p.rows = rows = p.blocks > 1 ? 8 : rows;
  // the shortest stretch, in places (3 and 6 were no better from 300 to 4000 keys)
  p.min_tiles = 4;
  p.nsplit = 1;
  // Tiles of 256 keys (8-bit pages of 64 channels): a chain for four 16-key groups instead
  // of two.  Up to 8 rows: 512 groups of 300 keys take 22.5 us so and 21.0 with 128, of 600 24.1
  // and 24.5, of 4000 61.7 and 75.1; shared out, 4 groups of 4000 9.9 and 9.4, 32 11.8 and 12.3.  9 to 16
  // rows: 512 of 1000 37.7 and 33.0, of 2500 53.9 and 57.0, 32 of 4000 14.3 and 13.9.
  const int64_t load = p.groups * max_visible;
  p.wide = codes && D == 64 && (rows <= 8 ? max_visible > 500 && (max_visible <= 2500 || load > 40000)
                                          : max_visible > 2000 && load > 400000);
  const int64_t tiles = (max_visible + 63) / 64 + 1;                  // of 64 keys, of a group at most
  // Whole groups, a CTA each, take their waves x (a CTA's start and end and its
  // tiles), the line an even share of all places after its start, parts and join.
  // In us, fitted to 1 to 8 sequences of 64 to 2000 keys; a tile's time is its own
  // chain's, or its share of HBM when many CTAs stream.  Long groups are shared:
  // they seldom have one length.  More groups than counters fill the SMs uncut.
  // 12 groups of 1000 keys of 128 channels take 8.8 us whole and 9.2 shared, of
  // 2000 keys 13.3 and 10.2; 48 of 1500 keys 11.2 and 13.0, of 2000 13.5 and 12.7;
  // 8 groups of 1000 keys of 64 channels 6.7 and 8.4.  Near the change the two are
  // close, and 96 groups of 2000 keys swing: 17 to 20 us either way.
  // 8-bit pages (4 to 320 groups of 130 to 4000 keys): 12 groups of 1000 keys of 128
  // channels 9.0 whole and 9.6 shared, of 1500 11.3 and 10.1; 96 of 2000 14.5 and 15.9; 192 of 1500
  // 24.0 and 23.8; of 64 channels 48 of 2000 11.1 and 10.7, 192 of 1000 14.6 and 17.2.
  struct Costs {
    double chain, hbm, start, line, place;   // a tile, a whole group's start; the line's start, a place
    int group;
  };
  const Costs u = p.wide ? Costs{0.16, 0.17, 4.4, 8.4, 0.19, 14}
                  : codes ? (D == 128 ? Costs{0.267, 0.308, 4.75, 8.6, 0.31, 12} : Costs{0.228, 0.24, 4.2, 8.0, 0.238, 14})
                        : (D == 128 ? Costs{0.29, 0.71, 4.0, 8.2, 0.44, group_cost<false>()}
                                    : Costs{0.24, 0.4, 2.8, 7.6, 0.33, group_cost<false>()});
  const double stream = p.groups < nsm ? u.hbm * p.groups / nsm : u.hbm;
  const double each = stream > u.chain ? stream : u.chain;
  const double whole = (double)((p.groups + nsm - 1) / nsm) * (u.start + tiles * each);
  const double shared = u.line + u.place * (double)(tiles + u.group) * p.groups / nsm;
  if (split && (tiles > 40 || whole > shared) && p.groups <= QWM_PAGED_COUNTER_BYTES / 4) {
    // a CTA per SM, or as many as have min_tiles places each
    const int tk = D == 128 && !codes ? 64 : (p.wide ? 256 : 128);
    if (p.wide) p.min_tiles = 3;
    const int64_t places = ((max_visible + tk - 1) / tk + 1 + (!codes ? group_cost<false>() : p.wide ? group_cost<true, 4>() : group_cost<true>())) * p.groups;
    const int64_t want = (places + p.min_tiles - 1) / p.min_tiles;
    p.nsplit = (int)(want < nsm ? want : nsm);
  }
  return p;
}

cudaError_t launch_paged_step(const PagedArgs& a, const CUtensorMap& map, int D, int dtype, cudaStream_t s) {
  if (dtype == QWM_F16) return D == 64 ? pick<__half, 64>(a, map, s) : pick<__half, 128>(a, map, s);
  return D == 64 ? pick<__nv_bfloat16, 64>(a, map, s) : pick<__nv_bfloat16, 128>(a, map, s);
}

}  // namespace qwm
