// Kernels over lists of arrays: the global norm of gradients, their scaling by a clipping coefficient, and the AdamW and Lion
// steps of parameters that are not matrices.
//
// One launch covers a whole list.  The arrays' descriptors travel in the launch's parameters (no table in device memory: nothing
// to copy before the launch, and a captured launch keeps its own).  The list is cut into tiles, numbered through; block b of G
// walks the tiles [T b / G, T (b + 1) / G), so every block has the same share whatever the arrays' sizes, finds its first array by
// one search and steps from array to array after that.
#pragma once

#include "dion_common.cuh"

namespace dion {
namespace list {

constexpr int THREADS = 256;
constexpr int NORM_RESIDENT = 4, SCALE_RESIDENT = 4, ADAMW_RESIDENT = 3, LION_RESIDENT = 4;      // blocks per SM
constexpr int TILE_UNITS = 256;      // vectors of a tile, one per thread
constexpr int TILE_SINGLES = 1024;   // elements of a tile that is walked one by one
constexpr int W = 8;                 // elements of a vector: 32 bytes of fp32 (one load on sm_100), 16 of bf16

// How an array is walked.
enum : int {
  SINGLES = 0,       // element by element: the pointers' alignments differ, or rows are no whole vectors
  DENSE = 1,         // one row: `head` elements up to the first 32-byte boundary, `units` vectors, the rest
  SLICED = 2         // rows of `cols` vectors, all aligned
};
struct Walk {
  i64 n, units, cols;            // elements; vectors (SINGLES: elements); of these in a row
  i64 first;                     // its first tile
  int head, kind;
};
struct NormItem {
  Walk w;
  const void* g;
  i64 ldg;
  int g_bf16;
};
struct ScaleItem {
  Walk w;
  const void* g;
  void* out;
  i64 ldg, ldo;
  int g_bf16, o_bf16;
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
  int g_bf16, m_bf16;
};

template <class Item, int CAP>
struct Table {
  i64 tiles;
  int count;
  Item item[CAP];
};

// What a norm launch leaves besides the caller's outputs (context scratch; its calls do not overlap).
struct Scratch {
  unsigned ticket;               // blocks that are done; zero between launches
  float coef;                    // clipping coefficient for the launch behind
  double carry;                  // sum (or maximum) over the launches of a list that takes several
  double pad[14];
  double part[1];                // one entry per block and array that it touches
};

struct NormOut {
  Scratch* scratch;
  float* norm;                   // optional: the total
  float* each;                   // optional: the norm of every array of this launch
  float* coef;                   // optional: min(1, max_norm / total)
  float max_norm;
  int use_carry, last;           // launches of one list: adds the carry of the one before; is the one that writes the total
  int* status;
};

struct Clip {
  const float* coef;             // the coefficient on the device, or, where it is NULL,
  const float* norms;            // the norms of parts of the whole, of which it is made
  int count, inf;
  float max_norm;
  float* norm_out;
  float* coef_out;
  int* status;
};

struct Rule {
  double beta1, beta2;
  float b1, c1, b2, c2, eps;     // beta and 1 - beta
  float inv1, inv2;              // 1 / (1 - beta^t), AdamW
  const int64_t* step_dev;       // where it is given, t is read there
  const float* scale;            // optional: the gradients' factor
  int first;                     // the first launch of a list: counts a cancelled step
  int* status;                   // [0] bits, [1] cancelled steps
};

template <class Table>
__device__ __forceinline__ int find_item(const Table& t, i64 tile) {      // the last array that starts at or before the tile
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.item[mid].w.first <= tile) lo = mid; else hi = mid - 1;
  }
  return lo;
}

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

// A block's part of one array, in vectors (elements, if it is walked one by one); `ends`: with the elements before and behind
// the vectors of a dense array.
struct Part {
  i64 u0, u1;
  bool head, tail;
};
__device__ __forceinline__ Part part_of(const Walk& w, i64 tile, i64 end) {
  const int per = w.kind == SINGLES ? TILE_SINGLES : TILE_UNITS;
  Part p;
  p.u0 = (tile - w.first) * per;
  p.u1 = (end - w.first) * per;
  p.tail = p.u1 >= w.units;
  if (p.tail) p.u1 = w.units;
  p.head = p.u0 == 0;
  return p;
}
// The row of vector u (of element u in an array that is walked one by one).
__device__ __forceinline__ i64 row_at(const Walk& w, i64 u) { return w.cols == w.units ? 0 : row_of(u, w.cols); }
// Calls f(index) for the elements of a dense array that are in no vector.
template <class F>
__device__ __forceinline__ void ends_of(const Walk& w, const Part& p, F f) {
  if (w.kind != DENSE) return;
  if (p.head && (int)threadIdx.x < w.head) f((i64)threadIdx.x);
  const i64 rest = w.head + w.units * W + threadIdx.x;
  if (p.tail && rest < w.n) f(rest);
}

// Sums in 64 bits: squares of fp32 values neither overflow nor vanish there.  A group's squares are added in fp32 first (a
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
__device__ __forceinline__ void norm_vectors(const NormItem& it, const Part& p, Acc<INF>& acc) {
  const T* g = reinterpret_cast<const T*>(it.g);
  const Walk& w = it.w;
  i64 u = p.u0 + threadIdx.x;
  if (w.kind == DENSE) {
    g += w.head;
    for (; u + 3 * THREADS < p.u1; u += 4 * THREADS) {      // four loads in flight per thread
      float x[4][W];
#pragma unroll
      for (int k = 0; k < 4; ++k) load_vec(g + (u + k * THREADS) * W, x[k]);
#pragma unroll
      for (int k = 0; k < 4; ++k) acc.add(x[k]);
    }
    for (; u < p.u1; u += THREADS) {
      float x[W];
      load_vec(g + u * W, x);
      acc.add(x);
    }
  } else {
    for (; u < p.u1; u += THREADS) {
      const i64 row = row_at(w, u);
      float x[W];
      load_vec(g + row * it.ldg + (u - row * w.cols) * W, x);
      acc.add(x);
    }
  }
}

template <bool INF>
__device__ __forceinline__ void norm_part(const NormItem& it, const Part& p, Acc<INF>& acc) {
  if (it.w.kind == SINGLES) {
    for (i64 e = p.u0 + threadIdx.x; e < p.u1; e += 4 * THREADS) {
      float x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const i64 f = e + k * THREADS, row = row_at(it.w, f);
        x[k] = f < p.u1 ? load_as_float(it.g, row * it.ldg + (f - row * it.w.cols), it.g_bf16) : 0.f;
      }
      acc.add(x);
    }
  } else if (it.g_bf16) {
    norm_vectors<INF, __nv_bfloat16>(it, p, acc);
  } else {
    norm_vectors<INF, float>(it, p, acc);
  }
  ends_of(it.w, p, [&](i64 e) { acc.add(load_as_float(it.g, e, it.g_bf16)); });
}

// Global norm: every block leaves its partial sums, the last one to finish adds them up in the order of the blocks.
// With `each` a block leaves one sum per array that it touches, at [block + array]: both grow along the tiles, so no two share an
// entry and those of one array are neighbours.
template <int CAP, bool INF>
__global__ void __launch_bounds__(THREADS, NORM_RESIDENT) k_list_norm(const __grid_constant__ Table<NormItem, CAP> t, const NormOut o) {
  __shared__ double red[THREADS / 32];
  __shared__ bool last;
  pdl_enter();
  const i64 G = gridDim.x, t0 = t.tiles * blockIdx.x / G, t1 = t.tiles * (blockIdx.x + 1) / G;
  const bool each = o.each != nullptr;
  Scratch* s = o.scratch;
  Acc<INF> acc;
  for (i64 tile = t0, i = t0 < t1 ? find_item(t, t0) : 0; tile < t1; ++i) {
    const NormItem& it = t.item[i];
    i64 end = i + 1 < t.count ? t.item[i + 1].w.first : t.tiles;
    if (end > t1) end = t1;
    if (end <= tile) continue;
    norm_part(it, part_of(it.w, tile, end), acc);
    if (each) {
      const Acc<INF> r = block_reduce(acc, red);
      if (threadIdx.x == 0) s->part[blockIdx.x + i] = r.kept();
      acc = Acc<INF>();
    }
    tile = end;
  }
  if (!each) {
    const Acc<INF> r = block_reduce(acc, red);
    if (threadIdx.x == 0) s->part[blockIdx.x] = r.kept();
  }
  __threadfence();
  if (threadIdx.x == 0) last = atomicAdd(&s->ticket, 1u) == gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  __threadfence();
  Acc<INF> all;
  if (each) {
    // a warp per array: its first and last block are those that own its first and last tile
    for (int i = threadIdx.x >> 5; i < t.count; i += THREADS / 32) {
      const i64 f = t.item[i].w.first, l = (i + 1 < t.count ? t.item[i + 1].w.first : t.tiles) - 1;
      Acc<INF> a;
      if (f <= l) {
        const i64 b0 = ((f + 1) * G - 1) / t.tiles, b1 = ((l + 1) * G - 1) / t.tiles;
        for (i64 b = b0 + (threadIdx.x & 31); b <= b1; b += 32) a.merge(__ldcg(&s->part[b + i]));
      }
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        if (INF) a.m = max(a.m, __shfl_xor_sync(0xffffffffu, a.m, d));
        else a.s += __shfl_xor_sync(0xffffffffu, a.s, d);
      }
      if ((threadIdx.x & 31) == 0) { o.each[i] = a.norm(); all.merge(a.kept()); }
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

template <typename TG, typename TO, int N>
__device__ __forceinline__ void scale_some(const TG* g, TO* out, float coef) {      // N vectors, THREADS apart
  float x[N][W];
#pragma unroll
  for (int k = 0; k < N; ++k) load_vec(g + k * THREADS * W, x[k]);
#pragma unroll
  for (int k = 0; k < N; ++k) {
#pragma unroll
    for (int q = 0; q < W; ++q) x[k][q] *= coef;
    store_vec(out + k * THREADS * W, x[k]);
  }
}

template <typename TG, typename TO>
__device__ __forceinline__ void scale_vectors(const ScaleItem& it, const Part& p, float coef) {
  const TG* g = reinterpret_cast<const TG*>(it.g);
  TO* out = reinterpret_cast<TO*>(it.out);
  i64 u = p.u0 + threadIdx.x;
  if (it.w.kind == DENSE) {
    g += it.w.head;
    out += it.w.head;
    for (; u + 3 * THREADS < p.u1; u += 4 * THREADS) scale_some<TG, TO, 4>(g + u * W, out + u * W, coef);
    for (; u < p.u1; u += THREADS) scale_some<TG, TO, 1>(g + u * W, out + u * W, coef);
  } else {
    for (; u < p.u1; u += THREADS) {
      const i64 row = row_at(it.w, u), col = (u - row * it.w.cols) * W;
      scale_some<TG, TO, 1>(g + row * it.ldg + col, out + row * it.ldo + col, coef);
    }
  }
}

// out = coefficient * G.  Where G itself would be multiplied by one nothing is read or written.
template <int CAP>
__global__ void __launch_bounds__(THREADS, SCALE_RESIDENT) k_list_scale(const __grid_constant__ Table<ScaleItem, CAP> t, const Clip c) {
  __shared__ double red[THREADS / 32];
  __shared__ float shared_coef;
  pdl_enter();
  float coef;
  if (c.coef != nullptr) {
    coef = *c.coef;
  } else {
    Acc<false> sum;
    Acc<true> top;
    for (int k = threadIdx.x; k < c.count; k += THREADS) {
      const float x = c.norms[k];
      if (c.inf) top.add(x); else sum.add(x);
    }
    float norm;
    if (c.inf) norm = block_reduce(top, red).norm(); else norm = block_reduce(sum, red).norm();
    if (threadIdx.x == 0) {
      shared_coef = clip_coef(norm, c.max_norm);
      if (blockIdx.x == 0) {
        if (!isfinite(norm)) atomicOr(c.status, DION_STATUS_NONFINITE);
        if (c.norm_out != nullptr) *c.norm_out = norm;
        if (c.coef_out != nullptr) *c.coef_out = shared_coef;
      }
    }
    __syncthreads();
    coef = shared_coef;
  }
  // the last blocks of the list first: what the norm's launch read last is still in L2
  const i64 G = gridDim.x, b = G - 1 - blockIdx.x, t0 = t.tiles * b / G, t1 = t.tiles * (b + 1) / G;
  for (i64 tile = t0, i = t0 < t1 ? find_item(t, t0) : 0; tile < t1; ++i) {
    const ScaleItem& it = t.item[i];
    i64 end = i + 1 < t.count ? t.item[i + 1].w.first : t.tiles;
    if (end > t1) end = t1;
    if (end <= tile) continue;
    if (!(coef == 1.f && it.g == it.out)) {
      const Part p = part_of(it.w, tile, end);
      if (it.w.kind == SINGLES) {
        for (i64 e = p.u0 + threadIdx.x; e < p.u1; e += THREADS) {
          const i64 row = row_at(it.w, e), col = e - row * it.w.cols;
          store_as(it.out, row * it.ldo + col, it.o_bf16, coef * load_as_float(it.g, row * it.ldg + col, it.g_bf16));
        }
      } else if (it.g_bf16) {
        if (it.o_bf16) scale_vectors<__nv_bfloat16, __nv_bfloat16>(it, p, coef); else scale_vectors<__nv_bfloat16, float>(it, p, coef);
      } else {
        if (it.o_bf16) scale_vectors<float, __nv_bfloat16>(it, p, coef); else scale_vectors<float, float>(it, p, coef);
      }
      ends_of(it.w, p, [&](i64 e) { store_as(it.out, e, it.o_bf16, coef * load_as_float(it.g, e, it.g_bf16)); });
    }
    tile = end;
  }
}

// sign(beta1 m + (1 - beta1) s g).  A fp32 evaluation is off by less than 2^-22 of the gradient's term (its three roundings and
// those of the factors) and 2^-23 of the sum; where the terms cancel further than 2^-20 the sum is taken in 64 bits.
__device__ __forceinline__ float lion_sign(const Rule& r, float m, float g, float s) {
  const float a = r.c1 * (s * g), c = fmaf(r.b1, m, a);
  if (fabsf(c) <= 9.5367432e-7f * fabsf(a)) {
    const double d = r.beta1 * (double)m + (1.0 - r.beta1) * ((double)s * (double)g);
    return d > 0.0 ? 1.f : d < 0.0 ? -1.f : 0.f;
  }
  return c > 0.f ? 1.f : c < 0.f ? -1.f : c;      // (a NaN stays one)
}

// One element's step.  m is the new moment before it is rounded to the array's type: only what is kept is rounded.
template <bool ADAMW>
__device__ __forceinline__ void step_element(const Rule& r, float inv1, float inv2, float s, float lr, float keep, float& x, float& m, float& v, float g) {
  if (ADAMW) {
    g *= s;
    m = fmaf(r.b1, m, r.c1 * g);
    v = fmaf(r.b2, v, r.c2 * (g * g));
    x = fmaf(-lr, (m * inv1) / (sqrtf(v * inv2) + r.eps), x * keep);
  } else {
    x = fmaf(-lr, lion_sign(r, m, g, s), x * keep);
    m = fmaf(r.b2, m, r.c2 * (s * g));
  }
}

template <bool ADAMW>
__device__ __forceinline__ void step_single(const StepItem& it, const Rule& r, float inv1, float inv2, float s, i64 row, i64 col) {
  const float g = load_as_float(it.G, row * it.ldg + col, it.g_bf16);
  float x = it.X[row * it.ldx + col], m = load_as_float(it.M, row * it.ldm + col, it.m_bf16), v = 0.f;
  if (ADAMW) v = it.V[row * it.ldv + col];
  step_element<ADAMW>(r, inv1, inv2, s, it.lr, it.keep, x, m, v, g);
  it.X[row * it.ldx + col] = x;
  store_as(it.M, row * it.ldm + col, it.m_bf16, m);
  if (ADAMW) it.V[row * it.ldv + col] = v;
  if (it.X16 != nullptr) it.X16[row * it.ldx16 + col] = __float2bfloat16_rn(x);
}

template <bool ADAMW, typename TG, typename TM>
__device__ __forceinline__ void step_vector(const StepItem& it, const Rule& r, float inv1, float inv2, float s, float* px, const TG* pg, TM* pm, float* pv, __nv_bfloat16* p16) {
  float x[W], m[W], v[W], g[W];
  load_vec(pg, g);
  load_vec(pm, m);
  if (ADAMW) load_vec(pv, v);
  load_vec(px, x);
#pragma unroll
  for (int k = 0; k < W; ++k) {
    float none = 0.f;
    step_element<ADAMW>(r, inv1, inv2, s, it.lr, it.keep, x[k], m[k], ADAMW ? v[k] : none, g[k]);
  }
  store_vec(px, x);
  store_vec(pm, m);
  if (ADAMW) store_vec(pv, v);
  if (it.X16 != nullptr) store_vec(p16, x);
}

template <bool ADAMW, typename TG, typename TM>
__device__ __forceinline__ void step_vectors(const StepItem& it, const Part& p, const Rule& r, float inv1, float inv2, float s) {
  const TG* G = reinterpret_cast<const TG*>(it.G);
  TM* M = reinterpret_cast<TM*>(it.M);
  if (it.w.kind == DENSE) {
    for (i64 u = p.u0 + threadIdx.x; u < p.u1; u += THREADS) {
      const i64 e = it.w.head + u * W;
      step_vector<ADAMW>(it, r, inv1, inv2, s, it.X + e, G + e, M + e, it.V + e, it.X16 + e);
    }
  } else {
    for (i64 u = p.u0 + threadIdx.x; u < p.u1; u += THREADS) {
      const i64 row = row_at(it.w, u), col = (u - row * it.w.cols) * W;
      step_vector<ADAMW>(it, r, inv1, inv2, s, it.X + row * it.ldx + col, G + row * it.ldg + col, M + row * it.ldm + col, it.V + row * it.ldv + col, it.X16 + row * it.ldx16 + col);
    }
  }
}

template <int CAP, bool ADAMW>
__global__ void __launch_bounds__(THREADS, ADAMW ? ADAMW_RESIDENT : LION_RESIDENT) k_list_step(const __grid_constant__ Table<StepItem, CAP> t, const Rule r) {
  __shared__ float corr[2];
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
  const i64 G = gridDim.x, t0 = t.tiles * blockIdx.x / G, t1 = t.tiles * (blockIdx.x + 1) / G;
  for (i64 tile = t0, i = t0 < t1 ? find_item(t, t0) : 0; tile < t1; ++i) {
    const StepItem& it = t.item[i];
    i64 end = i + 1 < t.count ? t.item[i + 1].w.first : t.tiles;
    if (end > t1) end = t1;
    if (end <= tile) continue;
    const Part p = part_of(it.w, tile, end);
    if (it.w.kind == SINGLES) {
      for (i64 e = p.u0 + threadIdx.x; e < p.u1; e += THREADS) {
        const i64 row = row_at(it.w, e);
        step_single<ADAMW>(it, r, inv1, inv2, s, row, e - row * it.w.cols);
      }
    } else if (it.g_bf16) {
      if (it.m_bf16) step_vectors<ADAMW, __nv_bfloat16, __nv_bfloat16>(it, p, r, inv1, inv2, s);
      else step_vectors<ADAMW, __nv_bfloat16, float>(it, p, r, inv1, inv2, s);
    } else {
      if (it.m_bf16) step_vectors<ADAMW, float, __nv_bfloat16>(it, p, r, inv1, inv2, s);
      else step_vectors<ADAMW, float, float>(it, p, r, inv1, inv2, s);
    }
    ends_of(it.w, p, [&](i64 e) { step_single<ADAMW>(it, r, inv1, inv2, s, 0, e); });
    tile = end;
  }
}

}  // namespace list
}  // namespace dion
