// paged.cuh -- shared definitions of the paged storage's kernels: arguments,
// what a row sees, element types.
#pragma once

#include "qwm_internal.cuh"
#include "ptx_sm103.cuh"

namespace qwm {

// ------------------------------------------------------------ rope and append
struct RopeSegment {            // a tensor [N][heads][D] and where its rows go
  const void* src;
  void* dst;
  int32_t s_tok, s_head;        // strides in elements
  int32_t d_tok, d_head;
  int32_t heads;
  int32_t rotate;               // 0: copied
  int32_t page;                 // -1: to dst; 0 / 1: to the Keys / Values of the token's page
};
struct RopeArgs {
  RopeSegment seg[3];
  int32_t nseg, total_heads;
  int32_t D, pairs[3], P;
  float sign;                   // -1: the gradient
  int64_t N;
  const float* inv_freq;        // [P]; null: nothing is rotated
  const int32_t* pos;           // [N][3]
  // paged destinations
  const int32_t *q_off, *kv_len, *table;
  int32_t B, table_stride, page_log2, kv_heads, max_q, max_kv;
  int64_t num_pages;
  void* pages;
  int32_t* status;
};
cudaError_t launch_rope(const RopeArgs& a, int dtype, bool interleaved, cudaStream_t s);

// ------------------------------------------------------------ attention
struct PagedArgs {
  const void* q;
  void* out;
  int64_t q_tok, q_head, o_tok, o_head;  // strides in elements
  float* lse;                            // [Hq][N] or null
  int64_t N;
  const int32_t *q_off, *kv_len, *table;
  int32_t B, table_stride, max_q, max_kv;
  int32_t Hk, G;                         // cache heads, Query heads per cache head
  int32_t page_log2;
  int64_t num_pages;
  const void* pages;
  int32_t block, window, sinks;
  float scale;
  int32_t* status;
  uint64_t wait_ns;
  int32_t idle;                          // nonzero: the producers load nothing (test hook)
  // split along the keys.  chunk: at most nsplit parts of a group, of at least
  // min_tiles tiles; step: nsplit CTAs share the line of all tiles, at least
  // min_tiles places each.  nsplit 1: no split
  int32_t nsplit, min_tiles;
  float* part_o;                         // chunk [group][nsplit][D / 4][row][4]; step [CTA][2][row][D]
  float2* part_ml;                       // running (max, sum): chunk [group][nsplit][row], the maximum as the
                                         // power that P is taken against; step [CTA][2][row]
  int32_t* counter;                      // step: [group], zero between calls
};

// Launch shape of an attention call: which kernel, and its split.
struct PagedPlan {
  int32_t step;      // 1: paged_step.cu, 0: paged_chunk.cu
  int32_t groups;    // (sequence, head, row tile) triples of the grid
  int32_t rows;      // rows of a group
  int32_t nsplit, min_tiles;
};
PagedPlan plan_step(int B, int Hk, int D, int rows, int64_t max_visible, int nsm, bool split);
PagedPlan plan_chunk(int B, int Hk, int64_t rows, int64_t max_visible, int nsm, bool split);
cudaError_t launch_paged_step(const PagedArgs& a, const CUtensorMap& map, int D, int dtype, cudaStream_t s);
cudaError_t launch_paged_chunk(const PagedArgs& a, const CUtensorMap& map, int D, int dtype, cudaStream_t s);
// Limit of the waits that let copies and MMAs in flight finish after another
// wait has run out, before a CTA gives up its shared memory and TMEM.
constexpr uint64_t kDrainNs = 1000000000ull;
// cudaFuncSetAttribute once per device for a kernel with dynamic shared memory
// (`done`: the caller's static).
template <class K>
inline cudaError_t allow_smem(K kernel, int bytes, bool (&done)[64]) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 0 && dev < 64 && done[dev]) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess && dev >= 0 && dev < 64) done[dev] = true;
  return e;
}
// A launch that may be set up while the kernel before it on the stream still
// runs (programmatic dependent launch).  Every thread of the kernel calls
// grid_begin() before its first access to global memory: it waits for that
// kernel's end, then lets the next one be set up.  Back to back this hides the
// launch and the start of a CTA, 1 to 2 us of a short step's 5 to 12.
template <class... P, class... A>
inline cudaError_t launch_ahead(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t s, A&&... args) {
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}
// Rows (Query tokens x Query heads per cache head) up to which a sequence goes
// to the step kernel.  With 16 rows of 128 channels it takes 67 us against the
// chunk kernel's 77 (one sequence of 131071 tokens, 4 cache heads), 20 against 16
// (4000 tokens); a step kernel with a second tile of 16 rows lost on nearly every
// length (24 rows: 88 against 79 us and 27 against 16).
constexpr int kStepRows = 16;

// Pages as rows of D channels, [num_pages * 2 * heads][page_tokens][D]: boxes of
// 64 channels x min(page_tokens, 64) tokens, 128-byte swizzle.
bool make_page_map(CUtensorMap* m, const void* pages, int64_t blocks, int page_tokens, int D, int dtype);

// ------------------------------------------------------------ device helpers
#ifdef __CUDACC__

// See launch_ahead.
__device__ __forceinline__ void grid_begin() {
  asm volatile("griddepcontrol.wait;\n\tgriddepcontrol.launch_dependents;" ::: "memory");
}

__device__ __forceinline__ void record_status(int32_t* status, int code) {
  if (status) atomicCAS(status, 0, code);
}

// Sequence b of the batch: its rows [q0, q0 + qn) and length kv, held to the
// ranges that the tensors and the page table have.  False: something was out, or the
// first sequence does not start at row 0 or the last one not end at N, so that rows are
// left out (their sequences are as good as ever).
struct Seq {
  int64_t q0;
  int32_t qn, kv;
};
template <class A>
__device__ __forceinline__ bool load_seq(const A& a, int b, Seq& s) {
  const int64_t q0 = a.q_off[b], q1 = a.q_off[b + 1];
  const int64_t kv = a.kv_len[b];
  int64_t cap = (int64_t)a.table_stride << a.page_log2;
  if (cap > a.max_kv) cap = a.max_kv;
  const bool ok = q0 >= 0 && q1 >= q0 && q1 <= a.N && q1 - q0 <= a.max_q && kv >= 0 && kv <= cap;
  s.q0 = ok ? q0 : 0;
  s.qn = ok ? (int32_t)(q1 - q0) : 0;
  s.kv = ok ? (int32_t)kv : 0;
  const int64_t left = (b == 0 ? q0 : 0) | (b == a.B - 1 ? a.N - q1 : 0);   // rows left out
  return ok && left == 0;
}

// The tokens a Query at token p sees: [0, min(sinks, hi)) and [lo, hi).
struct Span {
  int32_t lo, hi;
};
__device__ __forceinline__ Span row_span(int p, int kv, int block, int window) {
  Span r{0, 0};
  if (p < 0) return r;
  const int64_t e = ((int64_t)(p / block) + 1) * block;
  r.hi = (int)(e < kv ? e : kv);
  const int64_t lo = window > 0 ? e - window : 0;
  r.lo = lo < 0 ? 0 : (lo > r.hi ? r.hi : (int)lo);
  return r;
}

// What the rows of tokens p0 <= p <= p1 of a sequence see together, as a list
// of tiles of TK keys: the window's from its second tile on, its first tile (cut
// by the rows' windows), then tiles that hold first tokens before it (few keys).
// The first tile taken gives the running maxima their start, so it is one that
// the rows see whole where there is such a tile.  lo and hi of a row grow with its token, so the first and the last row bound
// all.
struct Tiles {
  int32_t lo_min, lo_max, hi_min, hi_max;  // over the rows; a row with p < 0 has hi = 0
  int32_t n_win, w_start, n;
};
template <int TK>
__device__ __forceinline__ Tiles make_tiles(int p0, int p1, int kv, int block, int window, int sinks) {
  Tiles t;
  const Span a = row_span(p0 < 0 ? 0 : p0, kv, block, window), b = row_span(p1, kv, block, window);
  t.lo_min = a.lo;
  t.hi_min = p0 < 0 ? 0 : a.hi;
  t.lo_max = b.lo;
  t.hi_max = b.hi;
  const int s_end = min(min(sinks, t.lo_min), t.hi_max);
  const int n_first = (s_end + TK - 1) / TK;
  t.w_start = max(t.lo_min / TK, n_first);
  t.n_win = max(0, (t.hi_max + TK - 1) / TK - t.w_start);
  t.n = t.hi_max == 0 ? 0 : t.n_win + n_first;
  return t;
}
__device__ __forceinline__ int tile_at(const Tiles& t, int i) {
  return i < t.n_win ? t.w_start + (i + 1 < t.n_win ? i + 1 : 0) : i - t.n_win;
}
__device__ __forceinline__ bool sees(int j, int lo, int hi, int sinks) { return j < hi && (j >= lo || j < sinks); }
// Whether some row of the tiles sees a token of [j0, j1).
__device__ __forceinline__ bool any_sees(const Tiles& t, int j0, int j1, int sinks) {
  return j0 < t.hi_max && (j1 > t.lo_min || j0 < sinks);
}
// Whether every row sees every token of [j0, j1).
__device__ __forceinline__ bool all_see(const Tiles& t, int j0, int j1, int sinks) {
  return j1 <= t.hi_min && (j0 >= t.lo_max || j1 <= sinks);
}

__device__ __forceinline__ float ex2f(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The two element types.
template <typename T>
struct Elem;
template <>
struct Elem<__nv_bfloat16> {
  static constexpr bool bf16 = true;
  static constexpr uint32_t kExp = 0x7F80u;  // exponent field: all ones in infinities and NaN
  // How far (as a power of two) P may grow before it is taken against a new maximum,
  // and the power below 1 that the largest P of a new maximum has.  P, l and O are
  // floating-point multiples of the same power, so only the types' ranges bound the
  // two.  Together they are 0: P never passes 1, and O holds every Value that an
  // ordinary sum holds (with P from 1 to 2^40 Values of 2^100 became infinite).  The
  // price is at the other end, where Values below 2^-86 leave fp32's normal range.
  // Less room costs time: 2^14 takes 66.2 us where 2^40 takes 63.3 (880 Queries x 12
  // heads over 17600 keys), 2^6 86.9.
  static constexpr int kTau = 40, kBias = 40;
  __device__ static __forceinline__ uint32_t pack(float a, float b) { return ptx::pack_bf16(a, b); }
  __device__ static __forceinline__ float2 unpack(uint32_t w) {
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  }
  __device__ static __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};
template <>
struct Elem<__half> {
  static constexpr bool bf16 = false;
  static constexpr uint32_t kExp = 0x7C00u;
  static constexpr int kTau = 14, kBias = 0;  // P at most 65504; O has fp32's range above that
  __device__ static __forceinline__ uint32_t pack(float a, float b) { return ptx::pack_f16(a, b); }
  __device__ static __forceinline__ float2 unpack(uint32_t w) {
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
  }
  __device__ static __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};
// Whether a word of two elements holds an infinity or a NaN.
template <typename T>
__device__ __forceinline__ bool nonfinite2(uint32_t w) {
  const uint32_t lo = w & Elem<T>::kExp, hi = (w >> 16) & Elem<T>::kExp;
  return lo == Elem<T>::kExp || hi == Elem<T>::kExp;
}

#endif  // __CUDACC__

}  // namespace qwm
