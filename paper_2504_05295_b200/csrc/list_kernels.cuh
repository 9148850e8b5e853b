// Kernels over lists of arrays: the global norm of gradients, their scaling by a clipping coefficient, and the AdamW and Lion
// steps of parameters that are not matrices.
//
// One launch covers a whole list.  The arrays' descriptors travel in the launch's parameters (no table in device memory: nothing
// to copy before the launch, and a captured launch keeps its own).  The list is cut into tiles, numbered through; every block
// takes the same number of neighbouring tiles (or one more), whatever the arrays' sizes, finds its first array by one search and
// steps from array to array after that.
#pragma once

#include "dion_common.cuh"

namespace dion {
namespace list {

constexpr int THREADS = 256;
constexpr int NORM_RESIDENT = 4, SCALE_RESIDENT = 4, ADAMW_RESIDENT = 3, LION_RESIDENT = 4;      // blocks per SM
constexpr int MOST_NORM_BLOCKS = 1024, MOST_ARRAYS = 500, MOST_PARTS = MOST_NORM_BLOCKS + MOST_ARRAYS;      // of a norm launch
constexpr int FEW_PARTS = 8;         // partial results of an array that one thread adds up
constexpr int TILE_UNITS = 256;      // groups of a tile, one per thread
constexpr int BATCH = 4;             // elements that a thread takes at once from an array that is walked one by one
constexpr int W = 8;                 // elements of a group: 32 bytes of fp32 (one load on sm_100), 16 of bf16

// How an array is walked.  Its rows are cut into groups of W elements at multiples of W elements of the ADDRESS, which is the same
// cut for all arrays of an item: what lies wholly in its row is one access per array, what hangs over a row's end goes element
// by element.  A row of `width` elements has groups at up to (width + 14) / 8 places, and each row is given that many.
// The cut is that of the arrays that are written; a gradient that lies apart from them modulo W (or has another leading
// dimension) is read by the element, out of L1 after the first of a group (67M parameters, gradient in bf16: AdamW 587 us one
// by one, 258 so; scaling into another buffer 315 and 62).
// One by one go items whose written arrays do not agree, and narrow rows, most of whose groups would hang over an end.
struct Walk {
  i64 first;                     // its first tile
  i64 units, per_row;            // groups, or elements; of these in a row
  i64 width;                     // columns (of a dense array, which is one row: all elements)
  uint8_t phase, shift;          // address of row 0 and leading dimension, in elements modulo W
  bool singles;                  // one by one
  bool g_bf16, other_bf16;       // types: of G; of the result or the moment
  bool g_apart;                  // G is not cut as the others are
};
struct NormItem {
  Walk w;
  const void* g;
  i64 ldg;
};
struct ScaleItem {
  Walk w;
  const void* g;
  void* out;
  i64 ldg, ldo;
};
struct StepItem {
  Walk w;
  float* X;
  const void* G;
  void* M;
  float* V;
  __nv_bfloat16* X16;
  i64 ldx, ldg, ldm, ldv, ldx16;
  float lr, keep;                // lr * lr_scale; 1 - lr * lr_scale * weight_decay
};

template <class Item, int CAP>
struct Table {
  i64 tiles, per, rem;           // tiles; block b takes `per` of them, and one more where b < rem
  int count;
  Item item[CAP];
};

// What a norm launch leaves besides the caller's outputs (context scratch; its calls do not overlap).
// Indexes found in it are in bounds whatever launch wrote them.
struct Scratch {
  unsigned ticket;               // blocks that are done; zero between launches
  float coef;                    // clipping coefficient for the launch behind
  double carry;                  // sum (or maximum) over the launches of a list that takes several
  double pad[14];
  int from[MOST_ARRAYS], upto[MOST_ARRAYS];      // with norms of each: an array's entries of `part`; zero between launches
  double part[MOST_PARTS];       // one entry per block and array that it touches
};

struct NormOut {
  Scratch* scratch;
  float* norm;                   // optional: the total
  float* each;                   // optional: the norm of every array of this launch
  float* coef;                   // optional: min(1, max_norm / total)
  float max_norm;
  int leave;                     // without `each`: the blocks' sums are left to the launch behind, which adds them up
  int use_carry, last;           // launches of one list: adds the carry of the one before; is the one that writes the total
  int* status;
};

struct Clip {
  const float* coef;             // the coefficient on the device, or what it is made of:
  const double* sums;            // what the blocks of a norm's launch left, or
  const float* norms;            // the norms of parts of the whole,
  int count, inf;                // and how many; which norm
  int in_place;                  // every array of the launch
  float max_norm;
  float* norm_out;
  float* coef_out;
  int* status;
};

// A beta in two parts, hi + lo within 2^-47 of it.  Rounded to fp32 alone it is off by as much as the rounding of a state, but the
// same way in every step: V would settle 1.7e-4 off for beta2 = 0.9999, 1.4e-3 for 0.99999.  lo is above zero (unless beta is zero or
// next to it), so that an infinite state stays infinite.
struct Beta {
  float hi, lo;
};
struct Rule {
  double beta1, beta2;
  Beta m, v;                     // of the moment and of AdamW's second one
  float b1, c1, cm, cv, eps;     // Lion's sign: beta1 and 1 - beta1; 1 - beta of the moment and of AdamW's second one
  float inv1, inv2;              // 1 / (1 - beta^t), AdamW
  const int64_t* step_dev;       // where it is given, t is read there
  const float* scale;            // optional: the gradients' factor
  int first;                     // the first launch of a list: counts a cancelled step
  int* status;                   // [0] bits, [1] cancelled steps
};

// The first tile of block b.
template <class Table>
__device__ __forceinline__ i64 first_tile(const Table& t, i64 b) { return b * t.per + (b < t.rem ? b : t.rem); }
// The last array that starts at or before the tile.  Seven looks at a time: a look at the parameters is a round trip to memory
// the first time, and these do not wait for one another.
template <class Table>
__device__ __forceinline__ int find_item(const Table& t, i64 tile) {
  int lo = 0;
  for (int span = t.count > 64 ? 64 : t.count > 8 ? 8 : 1; span > 0; span /= 8) {
    int ahead = 0;
#pragma unroll
    for (int k = 1; k < 8; ++k) {
      const int at = lo + k * span;
      if (at < t.count && t.item[at].w.first <= tile) ahead = k;
    }
    lo += ahead * span;
  }
  return lo;
}
static_assert(8 * 64 >= MOST_ARRAYS, "find_item reaches every array of a table");

__device__ __forceinline__ float load_as_float(const void* p, i64 at, int bf16) {
  return bf16 ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[at]) : reinterpret_cast<const float*>(p)[at];
}
__device__ __forceinline__ void store_as(void* p, i64 at, int bf16, float v) {
  if (bf16) reinterpret_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(v);
  else reinterpret_cast<float*>(p)[at] = v;
}

// Eight elements in one access: fp32 32 bytes, bf16 16.  Everything is touched once: not kept in L1.
__device__ __forceinline__ void load_vec(const float* p, float (&x)[W]) {
  asm volatile("ld.global.L1::no_allocate.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]) : "l"(p));
}
__device__ __forceinline__ void load_vec(const __nv_bfloat16* p, float (&x)[W]) {
  uint32_t r[4];
  asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "l"(p));
#pragma unroll
  for (int k = 0; k < 4; ++k) { x[2 * k] = __uint_as_float(r[k] << 16); x[2 * k + 1] = __uint_as_float(r[k] & 0xffff0000u); }
}
__device__ __forceinline__ void store_vec(float* p, const float (&x)[W]) {
  asm volatile("st.global.L1::no_allocate.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               :: "l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]) : "memory");
}
__device__ __forceinline__ void store_vec(__nv_bfloat16* p, const float (&x)[W]) {
  uint32_t r[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * k], x[2 * k + 1]);
    r[k] = *reinterpret_cast<const uint32_t*>(&v);
  }
  asm volatile("st.global.L1::no_allocate.v4.b32 [%0], {%1,%2,%3,%4};" :: "l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}

// Elements lo to hi of a group, where p points to its (perhaps missing) element 0.
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_float(float* p, float x) { *p = x; }
__device__ __forceinline__ void from_float(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }
template <typename T>
__device__ __forceinline__ void load_part(const T* p, float (&x)[W], int lo, int hi) {
#pragma unroll
  for (int k = 0; k < W; ++k) x[k] = k >= lo && k < hi ? to_float(p[k]) : 0.f;
}
template <typename T>
__device__ __forceinline__ void store_part(T* p, const float (&x)[W], int lo, int hi) {
#pragma unroll
  for (int k = 0; k < W; ++k)
    if (k >= lo && k < hi) from_float(p + k, x[k]);
}
template <typename T>
__device__ __forceinline__ void load_group(const T* p, float (&x)[W], int lo, int hi) {
  if (lo == 0 && hi == W) load_vec(p, x); else load_part(p, x, lo, hi);
}
template <typename T>
__device__ __forceinline__ void load_gradient(const T* p, float (&x)[W], int lo, int hi, bool apart) {
  if (lo == 0 && hi == W && !apart) load_vec(p, x); else load_part(p, x, lo, hi);
}
template <typename T>
__device__ __forceinline__ void store_group(T* p, const float (&x)[W], int lo, int hi) {
  if (lo == 0 && hi == W) store_vec(p, x); else store_part(p, x, lo, hi);
}

// A block's part of one array, in groups or elements.
struct Part {
  i64 u0, u1;
};
__device__ __forceinline__ Part part_of(const Walk& w, i64 tile, i64 end) {
  const int per = w.singles ? THREADS * BATCH : TILE_UNITS;
  Part p;
  p.u0 = (tile - w.first) * per;
  p.u1 = (end - w.first) * per;
  if (p.u1 > w.units) p.u1 = w.units;
  return p;
}
// Row and column of group u's element 0, and which of its elements exist; of element u in an array that is walked one by one.
struct Spot {
  i64 row, col;
  int lo, hi;
};
__device__ __forceinline__ i64 row_at(const Walk& w, i64 u) { return w.per_row == w.units ? 0 : row_of(u, w.per_row); }
__device__ __forceinline__ Spot group_at(const Walk& w, i64 u) {
  Spot s;
  s.row = row_at(w, u);
  s.col = (u - s.row * w.per_row) * W - ((w.phase + (uint32_t)s.row * w.shift) & (W - 1));
  s.lo = s.col < 0 ? (int)-s.col : 0;
  s.hi = w.width - s.col < W ? (int)(w.width - s.col) : W;      // (below lo: a place that this row does not fill)
  return s;
}

template <int N>
struct Number {
  static constexpr int value = N;
};

// Of a block's part, the groups of one row: wide rows (and dense arrays, which are one) are walked row by row, since the arithmetic
// of group_at is several times that of a norm.  All groups are whole but the row's first (if the row starts inside one) and its
// last; `first` and `last` are theirs if the part has them, else -1.
constexpr int WIDE = THREADS;        // groups of a wide row
struct RowRun {
  i64 row, col;                      // the row, and the column of its group 0
  i64 lo, hi;                        // whole groups
  i64 first, last;
  i64 end;                           // of the part: where the next row goes on
};
__device__ __forceinline__ bool by_rows(const Walk& w) { return w.per_row >= WIDE || w.per_row == w.units; }
__device__ __forceinline__ RowRun row_run(const Walk& w, i64 u, i64 u1) {
  RowRun r;
  r.row = row_at(w, u);
  const i64 u0 = r.row * w.per_row, k0 = u - u0;
  r.end = u0 + w.per_row < u1 ? u0 + w.per_row : u1;
  const i64 k1 = r.end - u0, phase = (w.phase + (uint32_t)r.row * w.shift) & (W - 1), whole = (w.width + phase) / W;
  r.col = -phase;
  r.lo = k0 == 0 && phase != 0 ? 1 : k0;
  r.hi = k1 < whole ? k1 : whole;
  r.first = k0 == 0 && phase != 0 ? 0 : -1;
  r.last = whole >= r.lo && whole < k1 && whole * W < w.width + phase ? whole : -1;
  return r;
}
// The row's first group is thread 0's, its last one another's.
__device__ __forceinline__ i64 end_group(const RowRun& r) { return threadIdx.x == 0 ? r.first : threadIdx.x == 32 ? r.last : -1; }
__device__ __forceinline__ Spot spot_in(const Walk& w, const RowRun& r, i64 k) {
  Spot s;
  s.row = r.row;
  s.col = r.col + k * W;
  s.lo = s.col < 0 ? (int)-s.col : 0;
  s.hi = w.width - s.col < W ? (int)(w.width - s.col) : W;
  return s;
}

// Sums in 64 bits: squares of fp32 values neither overflow nor vanish there.  A group's eight squares are added in fp32 first (a
// conversion and a 64-bit operation per element would cost more than the memory: 436M x 4 bf16 elements 6566 us); a sum that left
// fp32's range, or came close enough to its lower end to have lost something, is taken again.  Maxima on the magnitudes'
// bits, whose order is that of the values with NaN above infinity, so that a NaN is never lost.
template <bool INF>
struct Acc {
  double s = 0.0;
  uint32_t m = 0;
  template <int N>
  __device__ __forceinline__ void add(const float (&x)[N]) {
    if (INF) {
#pragma unroll
      for (int k = 0; k < N; ++k) m = max(m, __float_as_uint(x[k]) & 0x7fffffffu);
      return;
    }
    float q = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k) q = fmaf(x[k], x[k], q);
    if (q >= 7.8886091e-31f && q <= 3.4028235e38f) {      // (2^-100: what is below 2^-149 in a square is nothing beside it)
      s += (double)q;
    } else {
      bool any = false;
#pragma unroll
      for (int k = 0; k < N; ++k) any |= x[k] != 0.f;
      if (any) {
#pragma unroll
        for (int k = 0; k < N; ++k) s += (double)x[k] * (double)x[k];
      }
    }
  }
  __device__ __forceinline__ void add(float x) { const float one[1] = {x}; add(one); }
  __device__ __forceinline__ void merge(double v) {        // a partial result as it is kept
    if (INF) m = max(m, __float_as_uint((float)v));
    else s += v;
  }
  __device__ __forceinline__ double kept() const { return INF ? (double)__uint_as_float(m) : s; }
  __device__ __forceinline__ float norm() const { return INF ? __uint_as_float(m) : (float)sqrt(s); }
};

// The block's result in thread 0, in an order that does not depend on timing.
template <bool INF>
__device__ __forceinline__ Acc<INF> block_reduce(Acc<INF> a, double* smem) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    if (INF) a.m = max(a.m, __shfl_xor_sync(0xffffffffu, a.m, d));
    else a.s += __shfl_xor_sync(0xffffffffu, a.s, d);
  }
  __syncthreads();      // the entries of an earlier call have been read
  if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = a.kept();
  __syncthreads();
  Acc<INF> r;
  if (threadIdx.x == 0)
    for (int w = 0; w < THREADS / 32; ++w) r.merge(smem[w]);
  return r;
}

__device__ __forceinline__ float clip_coef(float norm, float max_norm) {
  // (a norm that is no number spoils the gradients, so that every step that reads them sees it)
  return !isfinite(norm) ? __int_as_float(0x7fffffff) : norm > max_norm ? max_norm / norm : 1.f;
}

template <bool INF, typename T>
__device__ __forceinline__ void norm_groups(const NormItem& it, const Part& p, Acc<INF>& acc) {
  const T* g = reinterpret_cast<const T*>(it.g);
  const Walk& w = it.w;
  if (by_rows(w)) {
    for (i64 u = p.u0; u < p.u1;) {
      const RowRun r = row_run(w, u, p.u1);
      const T* g0 = g + r.row * it.ldg + r.col;
      i64 k = r.lo + threadIdx.x;
      for (; k + 3 * THREADS < r.hi; k += 4 * THREADS) {      // four loads in flight per thread
        float x[4][W];
#pragma unroll
        for (int q = 0; q < 4; ++q) load_vec(g0 + (k + q * THREADS) * W, x[q]);
#pragma unroll
        for (int q = 0; q < 4; ++q) acc.add(x[q]);
      }
      for (; k < r.hi; k += THREADS) {
        float x[W];
        load_vec(g0 + k * W, x);
        acc.add(x);
      }
      k = end_group(r);
      if (k >= 0) {
        const Spot s = spot_in(w, r, k);
        float x[W];
        load_part(g0 + k * W, x, s.lo, s.hi);
        acc.add(x);
      }
      u = r.end;
    }
    return;
  }
  for (i64 u = p.u0 + threadIdx.x; u < p.u1; u += THREADS) {
    const Spot s = group_at(w, u);
    float x[W];
    load_group(g + s.row * it.ldg + s.col, x, s.lo, s.hi);
    acc.add(x);
  }
}

template <bool INF>
__device__ __forceinline__ void norm_part(const NormItem& it, const Part& p, Acc<INF>& acc) {
  if (it.w.singles) {
    for (i64 e = p.u0 + threadIdx.x; e < p.u1; e += BATCH * THREADS) {
      float x[BATCH];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const i64 f = e + k * THREADS, row = row_at(it.w, f);
        x[k] = f < p.u1 ? load_as_float(it.g, row * it.ldg + (f - row * it.w.per_row), it.w.g_bf16) : 0.f;
      }
      acc.add(x);
    }
  } else if (it.w.g_bf16) {
    norm_groups<INF, __nv_bfloat16>(it, p, acc);
  } else {
    norm_groups<INF, float>(it, p, acc);
  }
}

// Global norm: every block leaves its partial sums, the last one to finish adds them up in the order of the blocks.
// With `each` a block leaves one sum per array that it touches, at [block + array]: both grow along the tiles, so no two share an
// entry and those of one array are neighbours.  The blocks that see an array begin and end note which they are.  (Finding that out
// from the descriptors at the end, and one warp after another for arrays of many parts, cost 65 odd slices 1.7 us of 9.3.)
template <int CAP, bool INF>
__global__ void __launch_bounds__(THREADS, NORM_RESIDENT) k_list_norm(const __grid_constant__ Table<NormItem, CAP> t, const NormOut o) {
  __shared__ double red[THREADS / 32];
  __shared__ bool last;
  __shared__ double parts[MOST_PARTS];
  __shared__ int from[CAP], upto[CAP], many[CAP], manies;
  __shared__ double sums[CAP];
  const i64 G = gridDim.x, t0 = first_tile(t, blockIdx.x), t1 = first_tile(t, blockIdx.x + 1);
  i64 i = t0 < t1 ? find_item(t, t0) : 0;
  pdl_enter();
  const bool each = o.each != nullptr;
  Scratch* s = o.scratch;
  Acc<INF> acc;
  for (i64 tile = t0; tile < t1; ++i) {
    const NormItem& it = t.item[i];
    const i64 next = i + 1 < t.count ? t.item[i + 1].w.first : t.tiles, end = next < t1 ? next : t1;
    if (end <= tile) continue;
    norm_part(it, part_of(it.w, tile, end), acc);
    if (each) {
      const Acc<INF> r = block_reduce(acc, red);
      if (threadIdx.x == 0) {
        const int slot = (int)(blockIdx.x + i);
        s->part[slot] = r.kept();
        if (tile == it.w.first) s->from[i] = slot;
        if (end == next) s->upto[i] = slot + 1;
      }
      acc = Acc<INF>();
    }
    tile = end;
  }
  if (!each) {
    const Acc<INF> r = block_reduce(acc, red);
    if (threadIdx.x == 0) s->part[blockIdx.x] = r.kept();
    if (o.leave) return;
  }
  if (threadIdx.x == 0) {      // (it alone has written)
    __threadfence();
    last = atomicAdd(&s->ticket, 1u) == gridDim.x - 1;
    __threadfence();
  }
  __syncthreads();
  if (!last) return;
  Acc<INF> all;
  if (each) {
    // everything in one round trip; then a thread adds up an array's few parts, a warp many
    if (threadIdx.x == 0) manies = 0;
    for (int k = threadIdx.x; k < G + t.count; k += THREADS) parts[k] = __ldcg(&s->part[k]);
    for (int i = threadIdx.x; i < t.count; i += THREADS) {
      from[i] = __ldcg(&s->from[i]);
      upto[i] = __ldcg(&s->upto[i]);      // (an empty array's are zero)
      s->from[i] = 0;
      s->upto[i] = 0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < t.count; i += THREADS) {
      if (upto[i] - from[i] > FEW_PARTS) { many[atomicAdd(&manies, 1)] = i; continue; }
      Acc<INF> a;
      for (int k = from[i]; k < upto[i]; ++k) a.merge(parts[k]);
      sums[i] = a.kept();
    }
    __syncthreads();
    for (int m = threadIdx.x >> 5; m < manies; m += THREADS / 32) {
      const int i = many[m];
      Acc<INF> a;
      for (int k = from[i] + (threadIdx.x & 31); k < upto[i]; k += 32) a.merge(parts[k]);
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        if (INF) a.m = max(a.m, __shfl_xor_sync(0xffffffffu, a.m, d));
        else a.s += __shfl_xor_sync(0xffffffffu, a.s, d);
      }
      if ((threadIdx.x & 31) == 0) sums[i] = a.kept();
    }
    __syncthreads();
    for (int i = threadIdx.x; i < t.count; i += THREADS) {
      Acc<INF> a;
      a.merge(sums[i]);
      o.each[i] = a.norm();
      all.merge(sums[i]);
    }
  } else {
    for (i64 b = threadIdx.x; b < G; b += THREADS) all.merge(__ldcg(&s->part[b]));
  }
  all = block_reduce(all, red);
  if (threadIdx.x != 0) return;
  s->ticket = 0;
  if (o.use_carry) all.merge(s->carry);
  if (!o.last) { s->carry = all.kept(); return; }
  const float norm = all.norm();
  if (!isfinite(norm)) atomicOr(o.status, DION_STATUS_NONFINITE);
  const float coef = clip_coef(norm, o.max_norm);
  s->coef = coef;
  if (o.norm != nullptr) *o.norm = norm;
  if (o.coef != nullptr) *o.coef = coef;
}

// Short lists: norm and scaling in ONE launch of one cluster, the list in registers between the two.  A CTA has four teams of
// THREADS threads and a team up to KEPT tiles; the CTAs exchange their sums through shared memory of the cluster.  Bound by
// launches and round trips, not bytes; us per call from the host (in a graph), against two launches of the other kernels:
// clipping 2048 fp32 elements into bf16 5.7 (2.9) against 8.1 (5.3), 131072 5.6 (4.6) against 7.9 (5.9); the norm alone 2.8 against 3.5 and
// 3.4 against 4.2 in a graph.  At 262144, four tiles a team, it is 6.7 against 6.0 in a graph: eight SMs are too few by then.
constexpr int CLUSTER = 8, TEAMS = 4, KEPT = 3;
constexpr i64 CLUSTER_TILES = CLUSTER * TEAMS * KEPT;

template <int CAP, bool INF>
__global__ void __launch_bounds__(THREADS * TEAMS, 1) k_list_cluster(const __grid_constant__ Table<ScaleItem, CAP> t, const NormOut o, const int scale) {
  __shared__ double red[THREADS * TEAMS / 32];
  __shared__ double sums[CLUSTER];
  const int rank = blockIdx.x, team = threadIdx.x / THREADS, lane = threadIdx.x % THREADS;
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // (the others' shared memory is there once all have come)
  // tiles of this CTA, dealt to its teams in turn
  const i64 t0 = first_tile(t, rank), t1 = first_tile(t, rank + 1);
  int item[KEPT];
#pragma unroll
  for (int k = 0; k < KEPT; ++k) {
    const i64 tile = t0 + team + k * TEAMS;
    item[k] = tile < t1 ? find_item(t, tile) : -1;
  }
  pdl_enter();
  float x[KEPT][W];
  Acc<INF> acc;
#pragma unroll
  for (int k = 0; k < KEPT; ++k) {
#pragma unroll
    for (int q = 0; q < W; ++q) x[k][q] = 0.f;
    if (item[k] < 0) continue;
    const ScaleItem& it = t.item[item[k]];
    const i64 u = (t0 + team + k * TEAMS - it.w.first) * (it.w.singles ? THREADS * BATCH : TILE_UNITS) + lane;
    if (it.w.singles) {
#pragma unroll
      for (int q = 0; q < BATCH; ++q) {
        const i64 e = u + q * THREADS, row = row_at(it.w, e);
        if (e < it.w.units) x[k][q] = load_as_float(it.g, row * it.ldg + (e - row * it.w.per_row), it.w.g_bf16);
      }
    } else if (u < it.w.units) {
      const Spot at = group_at(it.w, u);
      const i64 e = at.row * it.ldg + at.col;
      if (it.w.g_bf16) load_gradient(reinterpret_cast<const __nv_bfloat16*>(it.g) + e, x[k], at.lo, at.hi, it.w.g_apart);
      else load_gradient(reinterpret_cast<const float*>(it.g) + e, x[k], at.lo, at.hi, it.w.g_apart);
    }
  }
#pragma unroll
  for (int k = 0; k < KEPT; ++k) acc.add(x[k]);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    if (INF) acc.m = max(acc.m, __shfl_xor_sync(0xffffffffu, acc.m, d));
    else acc.s += __shfl_xor_sync(0xffffffffu, acc.s, d);
  }
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = acc.kept();
  __syncthreads();
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  if (threadIdx.x < 32) {
    Acc<INF> a;
    a.merge(red[threadIdx.x]);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      if (INF) a.m = max(a.m, __shfl_xor_sync(0xffffffffu, a.m, d));
      else a.s += __shfl_xor_sync(0xffffffffu, a.s, d);
    }
    if (threadIdx.x < CLUSTER) {      // to every CTA of the cluster
      uint32_t to;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"((uint32_t)__cvta_generic_to_shared(&sums[rank])), "r"((uint32_t)threadIdx.x));
      asm volatile("st.shared::cluster.f64 [%0], %1;" :: "r"(to), "d"(a.kept()) : "memory");
    }
  }
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  Acc<INF> all;
#pragma unroll
  for (int k = 0; k < CLUSTER; ++k) all.merge(sums[k]);
  const float norm = all.norm(), coef = clip_coef(norm, o.max_norm);
  if (rank == 0 && threadIdx.x == 0) {
    if (!isfinite(norm)) atomicOr(o.status, DION_STATUS_NONFINITE);
    if (o.norm != nullptr) *o.norm = norm;
    if (o.coef != nullptr) *o.coef = coef;
  }
  if (!scale) return;
#pragma unroll
  for (int k = 0; k < KEPT; ++k) {
    if (item[k] < 0) continue;
    const ScaleItem& it = t.item[item[k]];
    if (coef == 1.f && it.g == it.out) continue;
    const i64 u = (t0 + team + k * TEAMS - it.w.first) * (it.w.singles ? THREADS * BATCH : TILE_UNITS) + lane;
#pragma unroll
    for (int q = 0; q < W; ++q) x[k][q] *= coef;
    if (it.w.singles) {
#pragma unroll
      for (int q = 0; q < BATCH; ++q) {
        const i64 e = u + q * THREADS, row = row_at(it.w, e);
        if (e < it.w.units) store_as(it.out, row * it.ldo + (e - row * it.w.per_row), it.w.other_bf16, x[k][q]);
      }
    } else if (u < it.w.units) {
      const Spot at = group_at(it.w, u);
      const i64 e = at.row * it.ldo + at.col;
      if (it.w.other_bf16) store_group(reinterpret_cast<__nv_bfloat16*>(it.out) + e, x[k], at.lo, at.hi);
      else store_group(reinterpret_cast<float*>(it.out) + e, x[k], at.lo, at.hi);
    }
  }
}

template <typename TG, typename TO, int N, bool APART = false>
__device__ __forceinline__ void scale_some(const TG* g, TO* out, float coef) {      // N groups, THREADS apart
  float x[N][W];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    if (APART) load_part(g + k * THREADS * W, x[k], 0, W); else load_vec(g + k * THREADS * W, x[k]);
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
#pragma unroll
    for (int q = 0; q < W; ++q) x[k][q] *= coef;
    store_vec(out + k * THREADS * W, x[k]);
  }
}

template <typename TG, typename TO>
__device__ __forceinline__ void scale_groups(const ScaleItem& it, const Part& p, float coef) {
  const TG* g = reinterpret_cast<const TG*>(it.g);
  TO* out = reinterpret_cast<TO*>(it.out);
  const Walk& w = it.w;
  const auto partly = [&](const Spot& s) {
    float x[W];
    load_gradient(g + s.row * it.ldg + s.col, x, s.lo, s.hi, w.g_apart);
#pragma unroll
    for (int k = 0; k < W; ++k) x[k] *= coef;
    store_group(out + s.row * it.ldo + s.col, x, s.lo, s.hi);
  };
  if (by_rows(w)) {      // as in norm_groups, but every row from its end
    for (i64 u = p.u0; u < p.u1;) {
      const RowRun r = row_run(w, u, p.u1);
      const TG* g0 = g + r.row * it.ldg + r.col;
      TO* out0 = out + r.row * it.ldo + r.col;
      if (w.g_apart) {
        for (i64 k = r.lo + threadIdx.x; k < r.hi; k += THREADS) scale_some<TG, TO, 1, true>(g0 + k * W, out0 + k * W, coef);
      } else {
        i64 fours = r.hi > r.lo ? r.lo + (r.hi - r.lo) / (4 * THREADS) * (4 * THREADS) : r.hi;
        for (i64 k = fours + threadIdx.x; k < r.hi; k += THREADS) scale_some<TG, TO, 1>(g0 + k * W, out0 + k * W, coef);
        while (fours > r.lo) {
          fours -= 4 * THREADS;
          scale_some<TG, TO, 4>(g0 + (fours + threadIdx.x) * W, out0 + (fours + threadIdx.x) * W, coef);
        }
      }
      const i64 k = end_group(r);
      if (k >= 0) partly(spot_in(w, r, k));
      u = r.end;
    }
    return;
  }
  for (i64 u = p.u0 + threadIdx.x; u < p.u1; u += THREADS) partly(group_at(w, u));
}

__device__ __forceinline__ void scale_singles(const ScaleItem& it, const Part& p, float coef) {
  for (i64 e = p.u0 + threadIdx.x; e < p.u1; e += BATCH * THREADS) {
    float x[BATCH];
    i64 row[BATCH];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const i64 f = e + k * THREADS;
      row[k] = row_at(it.w, f);
      x[k] = f < p.u1 ? load_as_float(it.g, row[k] * it.ldg + (f - row[k] * it.w.per_row), it.w.g_bf16) : 0.f;
    }
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const i64 f = e + k * THREADS;
      if (f < p.u1) store_as(it.out, row[k] * it.ldo + (f - row[k] * it.w.per_row), it.w.other_bf16, coef * x[k]);
    }
  }
}

// The norm of given norms, in every lane of every warp.
template <bool INF>
__device__ __forceinline__ float norm_of_norms(const Clip& c) {
  Acc<INF> a;
  for (int k = threadIdx.x & 31; k < c.count; k += 32) a.add(c.norms[k]);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    if (INF) a.m = max(a.m, __shfl_xor_sync(0xffffffffu, a.m, d));
    else a.s += __shfl_xor_sync(0xffffffffu, a.s, d);
  }
  return a.norm();
}

// The norm from the sums of a norm's blocks, in every thread: in the order in which that launch would have added them up.
template <bool INF>
__device__ __forceinline__ float norm_of_sums(const Clip& c, double* red, float* shared_norm) {
  Acc<INF> a;
  for (int k = threadIdx.x; k < c.count; k += THREADS) a.merge(__ldcg(c.sums + k));
  a = block_reduce(a, red);
  if (threadIdx.x == 0) *shared_norm = a.norm();
  __syncthreads();
  return *shared_norm;
}

// out = coefficient * G.  Where G itself would be multiplied by one nothing is read or written.
template <int CAP>
__global__ void __launch_bounds__(THREADS, SCALE_RESIDENT) k_list_scale(const __grid_constant__ Table<ScaleItem, CAP> t, const Clip c) {
  __shared__ double red[THREADS / 32];
  __shared__ float shared_norm;
  // What the norm's launch read last is still in L2: a block of one wave has the tiles that it had there and walks them from the
  // end; of many blocks those at the list's end come first.
  const i64 b = gridDim.x - 1 - blockIdx.x, t0 = first_tile(t, b), t1 = first_tile(t, b + 1);
  // (The search does not wait for the launch in front, except where the coefficient may say that nothing is to be done.  The loads of
  // G come behind the coefficient: where it is made of a norm's sums or of given norms, behind that reduction's barriers and shuffles.)
  i64 i = !c.in_place && t0 < t1 ? find_item(t, t1 - 1) : 0;
  pdl_enter();
  float coef;
  if (c.coef != nullptr) {
    coef = *c.coef;
  } else {
    const float norm = c.sums != nullptr ? (c.inf ? norm_of_sums<true>(c, red, &shared_norm) : norm_of_sums<false>(c, red, &shared_norm))
                                         : (c.inf ? norm_of_norms<true>(c) : norm_of_norms<false>(c));
    coef = clip_coef(norm, c.max_norm);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      if (!isfinite(norm)) atomicOr(c.status, DION_STATUS_NONFINITE);
      if (c.norm_out != nullptr) *c.norm_out = norm;
      if (c.coef_out != nullptr) *c.coef_out = coef;
    }
  }
  if (c.in_place) {
    if (coef == 1.f || t0 >= t1) return;
    i = find_item(t, t1 - 1);
  }
  for (i64 end = t1; end > t0; --i) {
    const ScaleItem& it = t.item[i];
    const i64 tile = it.w.first > t0 ? it.w.first : t0;
    if (tile >= end) continue;
    if (!(it.g == it.out && coef == 1.f)) {
      const Part p = part_of(it.w, tile, end);
      if (it.w.singles) {
        scale_singles(it, p, coef);
      } else if (it.w.g_bf16) {
        if (it.w.other_bf16) scale_groups<__nv_bfloat16, __nv_bfloat16>(it, p, coef); else scale_groups<__nv_bfloat16, float>(it, p, coef);
      } else {
        if (it.w.other_bf16) scale_groups<float, __nv_bfloat16>(it, p, coef); else scale_groups<float, float>(it, p, coef);
      }
    }
    end = tile;
  }
}

// sign(beta1 m + (1 - beta1) s g).  A fp32 evaluation is off by less than 2^-22 of the gradient's term (its three roundings and
// those of the factors), 2^-23 of the sum and, where a product falls below 2^-126, 2^-148; where the terms cancel further than
// 2^-20, and where the sum is below 2^-126, it is taken in 64 bits.
__device__ __forceinline__ float lion_sign(const Rule& r, float m, float g, float s) {
  const float a = r.c1 * (s * g), c = fmaf(r.b1, m, a);
  if (fabsf(c) <= fmaf(9.5367432e-7f, fabsf(a), 1.1754944e-38f)) {
    const double d = r.beta1 * (double)m + (1.0 - r.beta1) * ((double)s * (double)g);
    return d > 0.0 ? 1.f : d < 0.0 ? -1.f : 0.f;
  }
  return c > 0.f ? 1.f : c < 0.f ? -1.f : c;      // (a NaN stays one)
}

// The update's root and quotient need not be the nearest numbers (relative errors 2^-23 and 2^-22, of an update that is a
// thousandth of X or so); the correctly rounded ones are most of a short list's instructions (65 odd slices 11.9 us against 8.2).
// (Divisors: eps is 0 or between 2^-126 and 2^125, V's root 0 or between 2^-75 and 2^64, so their sum is below 2^-126 only as
// zero, where eps is, and below 2^126; or V is infinite and the quotient zero.)
__device__ __forceinline__ float sqrt_approx(float x) {
  float y;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float decayed(const Beta& b, float x, float c, float g) {      // beta x + c g
  return fmaf(b.hi, x, fmaf(b.lo, x, c * g));
}

// One element's step.  m is the new moment before it is rounded to the array's type: only what is kept is rounded.
template <bool ADAMW>
__device__ __forceinline__ void step_element(const Rule& r, float inv1, float inv2, float s, float lr, float keep, float& x, float& m, float& v, float g) {
  if (ADAMW) {
    g *= s;
    m = decayed(r.m, m, r.cm, g);
    v = decayed(r.v, v, r.cv, g * g);
    x = fmaf(-lr, __fdividef(m * inv1, sqrt_approx(v * inv2) + r.eps), x * keep);
  } else {
    x = fmaf(-lr, lion_sign(r, m, g, s), x * keep);
    m = decayed(r.m, m, r.cm, s * g);
  }
}

template <bool ADAMW>
__device__ __forceinline__ void step_singles(const StepItem& it, const Part& p, const Rule& r, float inv1, float inv2, float s) {
  for (i64 e = p.u0 + threadIdx.x; e < p.u1; e += BATCH * THREADS) {
    float x[BATCH], m[BATCH], v[BATCH], g[BATCH];
    i64 row[BATCH];
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {      // all loads first
      i64 f = e + k * THREADS;
      if (f >= p.u1) f = e;
      row[k] = row_at(it.w, f);
      const i64 col = f - row[k] * it.w.per_row;
      g[k] = load_as_float(it.G, row[k] * it.ldg + col, it.w.g_bf16);
      m[k] = load_as_float(it.M, row[k] * it.ldm + col, it.w.other_bf16);
      v[k] = ADAMW ? it.V[row[k] * it.ldv + col] : 0.f;
      x[k] = it.X[row[k] * it.ldx + col];
    }
#pragma unroll
    for (int k = 0; k < BATCH; ++k) {
      const i64 f = e + k * THREADS, col = f - row[k] * it.w.per_row;
      step_element<ADAMW>(r, inv1, inv2, s, it.lr, it.keep, x[k], m[k], v[k], g[k]);
      if (f >= p.u1) continue;
      it.X[row[k] * it.ldx + col] = x[k];
      store_as(it.M, row[k] * it.ldm + col, it.w.other_bf16, m[k]);
      if (ADAMW) it.V[row[k] * it.ldv + col] = v[k];
      if (it.X16 != nullptr) it.X16[row[k] * it.ldx16 + col] = __float2bfloat16_rn(x[k]);
    }
  }
}

template <bool ADAMW, typename TG, typename TM>
__device__ __forceinline__ void step_group(const StepItem& it, const Rule& r, float inv1, float inv2, float s, float* px, const TG* pg, TM* pm, float* pv,
                                           __nv_bfloat16* p16, int lo, int hi, bool apart) {
  float x[W], m[W], v[W], g[W];
  load_gradient(pg, g, lo, hi, apart);
  load_group(pm, m, lo, hi);
  if (ADAMW) load_group(pv, v, lo, hi);
  load_group(px, x, lo, hi);
#pragma unroll
  for (int k = 0; k < W; ++k) {
    float none = 0.f;
    step_element<ADAMW>(r, inv1, inv2, s, it.lr, it.keep, x[k], m[k], ADAMW ? v[k] : none, g[k]);
  }
  store_group(px, x, lo, hi);
  store_group(pm, m, lo, hi);
  if (ADAMW) store_group(pv, v, lo, hi);
  if (it.X16 != nullptr) store_group(p16, x, lo, hi);
}

// Dense arrays one by one.  (With the general form's addresses and types looked up for every element AdamW on 67M parameters whose
// written arrays lie apart takes 607 us, so 318; 258 where they agree.)
template <bool ADAMW, typename TG, typename TM>
__device__ __forceinline__ void step_dense(const StepItem& it, const Part& p, const Rule& r, float inv1, float inv2, float s) {
  float* X = it.X;
  const TG* G = reinterpret_cast<const TG*>(it.G);
  TM* M = reinterpret_cast<TM*>(it.M);
  float* V = it.V;
  __nv_bfloat16* X16 = it.X16;
  const float lr = it.lr, keep = it.keep;
  const auto some = [&](i64 e, auto count) {
    constexpr int N = decltype(count)::value;
    float x[N], m[N], v[N], g[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const i64 f = e + k * THREADS;
      g[k] = to_float(G[f]);
      m[k] = to_float(M[f]);
      v[k] = ADAMW ? V[f] : 0.f;
      x[k] = X[f];
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const i64 f = e + k * THREADS;
      step_element<ADAMW>(r, inv1, inv2, s, lr, keep, x[k], m[k], v[k], g[k]);
      X[f] = x[k];
      from_float(M + f, m[k]);
      if (ADAMW) V[f] = v[k];
      if (X16 != nullptr) X16[f] = __float2bfloat16_rn(x[k]);
    }
  };
  i64 e = p.u0 + threadIdx.x;
  for (; e + (BATCH - 1) * THREADS < p.u1; e += BATCH * THREADS) some(e, Number<BATCH>());
  for (; e < p.u1; e += THREADS) some(e, Number<1>());
}

template <bool ADAMW, typename TG, typename TM>
__device__ __forceinline__ void step_groups(const StepItem& it, const Part& p, const Rule& r, float inv1, float inv2, float s) {
  const TG* G = reinterpret_cast<const TG*>(it.G);
  TM* M = reinterpret_cast<TM*>(it.M);
  const Walk& w = it.w;
  const auto partly = [&](const Spot& at) {
    step_group<ADAMW>(it, r, inv1, inv2, s, it.X + at.row * it.ldx + at.col, G + at.row * it.ldg + at.col, M + at.row * it.ldm + at.col,
                      it.V + at.row * it.ldv + at.col, it.X16 + at.row * it.ldx16 + at.col, at.lo, at.hi, w.g_apart);
  };
  if (w.per_row == w.units) {      // one row: as in norm_groups.  (Other rows are bound by memory as they are.)
    const RowRun run = row_run(w, p.u0, p.u1);
    if (w.g_apart) {
      for (i64 k = run.lo + threadIdx.x; k < run.hi; k += THREADS) {
        const i64 e = k * W + run.col;
        step_group<ADAMW>(it, r, inv1, inv2, s, it.X + e, G + e, M + e, it.V + e, it.X16 + e, 0, W, true);
      }
    } else {
      for (i64 k = run.lo + threadIdx.x; k < run.hi; k += THREADS) {
        const i64 e = k * W + run.col;
        step_group<ADAMW>(it, r, inv1, inv2, s, it.X + e, G + e, M + e, it.V + e, it.X16 + e, 0, W, false);
      }
    }
    const i64 k = end_group(run);
    if (k >= 0) partly(spot_in(w, run, k));
    return;
  }
  for (i64 u = p.u0 + threadIdx.x; u < p.u1; u += THREADS) partly(group_at(w, u));
}

template <int CAP, bool ADAMW>
__global__ void __launch_bounds__(THREADS, ADAMW ? ADAMW_RESIDENT : LION_RESIDENT) k_list_step(const __grid_constant__ Table<StepItem, CAP> t, const Rule r) {
  __shared__ float corr[2];
  const i64 t0 = first_tile(t, blockIdx.x), t1 = first_tile(t, blockIdx.x + 1);
  i64 i = t0 < t1 ? find_item(t, t0) : 0;
  pdl_enter();
  const float s = r.scale != nullptr ? *r.scale : 1.f;
  if (!isfinite(s)) {
    if (blockIdx.x == 0 && threadIdx.x == 0 && r.first) {
      atomicOr(r.status, DION_STATUS_NONFINITE);
      atomicAdd(r.status + 1, 1);
    }
    return;
  }
  float inv1 = r.inv1, inv2 = r.inv2;
  if (ADAMW && r.step_dev != nullptr) {
    const i64 t_dev = *r.step_dev;
    if (t_dev < 1) {
      if (blockIdx.x == 0 && threadIdx.x == 0 && r.first) atomicAdd(r.status + 1, 1);
      return;
    }
    if (threadIdx.x == 0) {
      const double n = (double)t_dev;
      corr[0] = (float)(1.0 / (1.0 - pow(r.beta1, n)));
      corr[1] = (float)(1.0 / (1.0 - pow(r.beta2, n)));
    }
    __syncthreads();
    inv1 = corr[0]; inv2 = corr[1];
  }
  for (i64 tile = t0; tile < t1; ++i) {
    const StepItem& it = t.item[i];
    i64 end = i + 1 < t.count ? t.item[i + 1].w.first : t.tiles;
    if (end > t1) end = t1;
    if (end <= tile) continue;
    const Part p = part_of(it.w, tile, end);
    if (it.w.singles) {
      if (it.w.per_row != it.w.units) step_singles<ADAMW>(it, p, r, inv1, inv2, s);
      else if (it.w.g_bf16 && it.w.other_bf16) step_dense<ADAMW, __nv_bfloat16, __nv_bfloat16>(it, p, r, inv1, inv2, s);
      else if (it.w.g_bf16) step_dense<ADAMW, __nv_bfloat16, float>(it, p, r, inv1, inv2, s);
      else if (it.w.other_bf16) step_dense<ADAMW, float, __nv_bfloat16>(it, p, r, inv1, inv2, s);
      else step_dense<ADAMW, float, float>(it, p, r, inv1, inv2, s);
    } else if (it.w.g_bf16) {
      if (it.w.other_bf16) step_groups<ADAMW, __nv_bfloat16, __nv_bfloat16>(it, p, r, inv1, inv2, s);
      else step_groups<ADAMW, __nv_bfloat16, float>(it, p, r, inv1, inv2, s);
    } else {
      if (it.w.other_bf16) step_groups<ADAMW, float, __nv_bfloat16>(it, p, r, inv1, inv2, s);
      else step_groups<ADAMW, float, float>(it, p, r, inv1, inv2, s);
    }
    tile = end;
  }
}

}  // namespace list
}  // namespace dion
