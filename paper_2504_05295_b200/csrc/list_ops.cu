// Calls over lists of arrays: argument checks, the launches' descriptor tables, launches.
#include <math.h>
#include <stdlib.h>
#include <string.h>
#include <algorithm>
#include <new>
#include <numeric>
#include <type_traits>

#include "list_api.cuh"
#include "list_kernels.cuh"

namespace dion {
namespace list {

namespace {

// Blocks: one wave of resident ones (the kernels' launch bounds); of long lists more, each with a few tiles.  Blocks that start
// in order keep what is in flight close together in memory, and an SM that is slower takes fewer (AdamW on 268M parameters:
// 1249 us in one wave, 1238 with chunks dealt to one wave in turn, 1114 with 4 tiles a block, 1156 with 2; Lion 717, 647 with 4).
// Scaling 872M bf16 elements with their norm: 993 in one wave, 788, 796, 799, 813 with 8, 16, 24, 32 tiles; but where the
// coefficient is 1 every block is started for nothing: 1074M elements 307 us for the norm, 375, 342, 330, 325 with the launch behind it.
// One wave of scaling blocks has the tiles that the norm's blocks had, and finds the last of them in L2: 33.6M elements from fp32 to bf16
// 55.0 us against 59.1 with many blocks, bf16 to bf16 36.2 against 38.8; 67M 108.9 against 108.0 and 69.7 against 70.5.
struct Shape {
  int resident;             // blocks per SM of one wave,
  int tiles_one_wave;       // up to so many tiles a block,
  int tiles;                // and tiles of a block on longer lists
  i64 most;                 // blocks
};
constexpr i64 ANY = INT32_MAX;
constexpr Shape NORM_SHAPE = {NORM_RESIDENT, INT32_MAX, INT32_MAX, MOST_NORM_BLOCKS}, SCALE_SHAPE = {SCALE_RESIDENT, 64, 24, ANY},
                ADAMW_SHAPE = {ADAMW_RESIDENT, 4, 4, ANY}, LION_SHAPE = {LION_RESIDENT, 4, 4, ANY};
// Arrays in one launch: its parameters end at 32764 bytes.  A launch's parameters are copied whole (28 KB cost 3 us more than 7 KB), so
// tables come in four sizes.
constexpr int FEW = 24, SOME = 80, MORE = 180;
constexpr int MANY_NORM = 500, MANY_SCALE = 400, MANY_STEP = 250, MANY_CLUSTER = CLUSTER_TILES;
constexpr i64 MAX_ELEMENTS = (i64)1 << 50;      // (no element count or byte offset overflows)

// (The arguments by address: a typed launch would copy the table once more.)
template <typename... KArgs, typename... Args>
int launch_blocks(const Where& w, void (*kernel)(KArgs...), i64 blocks, int threads, int cluster, const Args&... args) {
  static_assert(sizeof...(KArgs) == sizeof...(Args) && (std::is_same<std::remove_cv_t<KArgs>, Args>::value && ...), "the kernel's own types");
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks); cfg.blockDim = dim3(threads); cfg.stream = w.stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = cluster > 1 ? 2 : 1;
  ++*w.launches;
  void* pointers[] = {const_cast<void*>((const void*)&args)...};
  if (cudaLaunchKernelExC(&cfg, (const void*)kernel, pointers) != cudaSuccess) { cudaGetLastError(); return DION_ERR_CUDA; }
  return DION_OK;
}

i64 blocks_for(const Where& w, const Shape& shape, i64 tiles) {
  i64 blocks = (i64)w.sm_count * shape.resident;
  if (tiles / shape.tiles_one_wave > blocks) blocks = tiles / shape.tiles;
  if (blocks > shape.most) blocks = shape.most;
  if (blocks > tiles) blocks = tiles;
  return blocks < 1 ? 1 : blocks;
}

template <class Table, typename... KArgs, typename... Args>
int launch(const Where& w, void (*kernel)(KArgs...), const Shape& shape, Table& t, const Args&... args) {
  const i64 blocks = blocks_for(w, shape, t.tiles);
  t.per = t.tiles / blocks; t.rem = t.tiles % blocks;
  return launch_blocks(w, kernel, blocks, THREADS, 1, t, args...);
}

inline int bytes_of(int dtype) { return dtype == DION_BF16 ? 2 : 4; }
inline bool known_type(int dtype) { return dtype == DION_F32 || dtype == DION_BF16; }

// rows x cols elements, or a refusal
bool too_many(i64 a, i64 b) { return ((a | b) >> 25) != 0 && (unsigned __int128)a * (unsigned __int128)b > (unsigned __int128)MAX_ELEMENTS; }
int check_shape(i64 rows, i64 cols) {
  return rows < 0 || cols < 0 || rows > MAX_ELEMENTS || cols > MAX_ELEMENTS || too_many(rows, cols) ? DION_ERR_SHAPE : DION_OK;
}
int check_array(const void* p, i64 rows, i64 cols, i64 ld, int size) {
  if (rows == 0 || cols == 0) return DION_OK;
  if (p == nullptr) return DION_ERR_INVALID;
  if (ld < cols || (rows > 1 && too_many(rows, ld))) return DION_ERR_SHAPE;
  return (uintptr_t)p & (uintptr_t)(size - 1) ? DION_ERR_ALIGN : DION_OK;
}

// Memory that a call reads or writes.  Rows of `width` bytes, `pitch` bytes apart.
struct Range {
  uintptr_t begin, end;
  uintptr_t width, pitch;      // pitch 0: one row
  uintptr_t rows;
  bool written;
};
Range range_of(const void* p, i64 rows, i64 cols, i64 ld, int size, bool written) {
  Range r;
  r.begin = (uintptr_t)p;
  r.width = (uintptr_t)(cols * size);
  r.pitch = rows > 1 && ld != cols ? (uintptr_t)(ld * size) : 0;
  if (r.pitch == 0) r.width = (uintptr_t)(rows * cols * size);
  r.rows = r.pitch == 0 ? 1 : (uintptr_t)rows;
  r.end = r.begin + (r.pitch == 0 ? r.width : (uintptr_t)(rows - 1) * r.pitch + r.width);
  r.written = written;
  return r;
}
// The first row of r that ends behind p.
uintptr_t row_behind(const Range& r, uintptr_t p) { return p < r.begin + r.width ? 0 : r.pitch == 0 ? 1 : (p - r.begin - r.width) / r.pitch + 1; }
// Whether any byte belongs to both.  The rows of one are looked up in the other, as far as the two lie beside one another: the
// first, which may begin before the other does, and as many more as begin at different places within the other's pitch.
bool conflict(const Range& a, const Range& b) {
  if ((!a.written && !b.written) || a.begin >= b.end || b.begin >= a.end) return false;
  const Range &x = b.pitch == 0 ? b : a, &y = b.pitch == 0 ? a : b;      // (if one of them is a single row, x is)
  const uintptr_t first = row_behind(x, y.begin), places = y.pitch == 0 ? 0 : y.pitch / std::gcd(x.pitch, y.pitch);
  for (uintptr_t i = first; i < x.rows && i - first <= places; ++i) {
    const uintptr_t from = x.begin + i * x.pitch;
    if (from >= y.end) break;
    if (y.begin + row_behind(y, from) * y.pitch < from + x.width) return true;      // (from < y.end: there is such a row)
  }
  return false;
}

// Ranges of one kind (all X, all G, ...), as runs of ranges that follow one another at once or after a short gap: lists are often
// views of a few buffers.
struct Run {
  uintptr_t begin, end;
};
class Runs {
 public:
  ~Runs() { if (run != few) delete[] run; }
  void add(const void* p, i64 rows, i64 cols, i64 ld, int size) {
    if (p == nullptr || rows == 0 || cols == 0) return;
    const uintptr_t b = (uintptr_t)p, e = b + (uintptr_t)((rows - 1) * ld + cols) * (uintptr_t)size;
    if (n > 0 && b >= run[n - 1].end && b - run[n - 1].end <= GAP) { run[n - 1].end = e; return; }
    if (n == cap && !grow()) return;
    sorted = sorted && (n == 0 || b >= run[n - 1].begin);
    run[n++] = {b, e};
  }
  void sort() {
    if (!sorted) std::sort(run, run + n, [](const Run& a, const Run& b) { return a.begin < b.begin; });
  }
  Run* run = few;
  int n = 0;
  bool no_memory = false;

 private:
  static constexpr uintptr_t GAP = 4096;
  bool grow() {
    Run* more = new (std::nothrow) Run[2 * (size_t)cap];
    if (more == nullptr) { no_memory = true; return false; }
    std::copy(run, run + n, more);
    if (run != few) delete[] run;
    run = more;
    cap *= 2;
    return true;
  }
  Run few[16];
  int cap = 16;
  bool sorted = true;
};

// Whether anything that a call writes is touched twice.  The kinds' runs are looked through side by side; where two of them meet,
// `each(f)` calls f(pointer, rows, cols, ld, size, written) for every range, and these are sorted and compared one by one.
template <int KINDS, class Each>
int check_ranges(Runs (&kind)[KINDS], const Each& each) {
  int at[KINDS] = {};
  bool apart = true;
  uintptr_t end = 0;
  for (Runs& k : kind) {
    if (k.no_memory) return DION_ERR_NOMEM;
    k.sort();
  }
  for (;;) {
    int first = -1;
    for (int k = 0; k < KINDS; ++k)
      if (at[k] < kind[k].n && (first < 0 || kind[k].run[at[k]].begin < kind[first].run[at[first]].begin)) first = k;
    if (first < 0) break;
    const Run& r = kind[first].run[at[first]++];
    if (r.begin < end) { apart = false; break; }
    end = r.end;
  }
  if (apart) return DION_OK;
  size_t n = 0;
  each([&](const void* p, i64 rows, i64 cols, i64, int, bool) { n += p != nullptr && rows != 0 && cols != 0; });
  Range* r = new (std::nothrow) Range[n];
  if (r == nullptr) return DION_ERR_NOMEM;
  n = 0;
  each([&](const void* p, i64 rows, i64 cols, i64 ld, int size, bool written) {
    if (p != nullptr && rows != 0 && cols != 0) r[n++] = range_of(p, rows, cols, ld, size, written);
  });
  std::sort(r, r + n, [](const Range& a, const Range& b) { return a.begin < b.begin; });
  int rc = DION_OK;
  for (size_t i = 0; i < n && rc == DION_OK; ++i)
    for (size_t j = i + 1; j < n && r[j].begin < r[i].end; ++j)
      if (conflict(r[i], r[j])) { rc = DION_ERR_ALIAS; break; }
  delete[] r;
  return rc;
}

bool norm_type_ok(int t) { return t == DION_NORM_2 || t == DION_NORM_INF; }

int check_floats(const float* p) { return (uintptr_t)p & 3 ? DION_ERR_ALIGN : DION_OK; }

#define LIST_TRY(expr)              \
  do {                              \
    const int rc_ = (expr);         \
    if (rc_ != DION_OK) return rc_; \
  } while (0)

// An array (of those that are walked together) as the walk needs it.
struct Array {
  const void* p;
  i64 ld;
  int shift;      // log2 of the element's bytes
};
inline int shift_of(int dtype) { return dtype == DION_BF16 ? 1 : 2; }

constexpr i64 NARROW = 32;      // rows of fewer elements go one by one

// How arrays of rows x cols are walked together, and their tiles behind the `tiles` so far.  The first of the arrays is the
// gradient, whose addresses need not agree with those of the others.
template <size_t N>
Walk plan(i64 rows, i64 cols, int g_dtype, int other_dtype, const Array (&a)[N], i64* tiles) {
  Walk w = {};
  w.first = *tiles;
  w.g_bf16 = g_dtype == DION_BF16; w.other_bf16 = other_dtype == DION_BF16;
  if (rows == 0 || cols == 0) return w;
  bool agree = true, dense = true;
  int phase = -1, shift = 0;
  for (size_t k = N; k-- > 0;) {
    const Array& x = a[k];
    if (x.p == nullptr) continue;
    const int ph = (int)((uintptr_t)x.p >> x.shift) & (W - 1), sh = (int)x.ld & (W - 1);
    const bool same = phase < 0 || (ph == phase && (rows == 1 || sh == shift));
    dense = dense && (rows == 1 || x.ld == cols);
    if (k == 0 && !same) { w.g_apart = true; break; }
    agree = agree && same;
    phase = ph; shift = sh;
  }
  if (dense) { cols *= rows; rows = 1; }
  w.width = cols;
  w.singles = !agree || (rows > 1 && cols < NARROW);
  if (w.singles) {
    w.per_row = cols;
  } else {
    // (one row's first group starts at its phase; the rows of a matrix start at any)
    w.per_row = rows == 1 ? (cols + phase + W - 1) / W : (cols + 2 * W - 2) / W;
    w.phase = (uint8_t)phase; w.shift = (uint8_t)(rows == 1 ? 0 : shift);
  }
  w.units = rows * w.per_row;
  const i64 per = w.singles ? THREADS * BATCH : TILE_UNITS;
  *tiles += (w.units + per - 1) / per;
  return w;
}

// Whether arrays that lie one behind the other can be walked as one: dense, of the same types, each where the one before it ends.
// Parameters and gradients are often views of flat buffers; 65 neighbours are one item instead of a table of 65 (AdamW, host
// time: 7.9 -> 6.6 us).
bool follows(const void* a, const void* b, i64 n, int size) { return (uintptr_t)b == (uintptr_t)a + (uintptr_t)(n * size); }
bool dense(const dion_grad& a, bool out) { return a.rows == 1 || (a.ldg == a.cols && (!out || a.ldo == a.cols)); }
bool continues(const dion_grad& a, const dion_grad& b, bool out) {
  const i64 n = a.rows * a.cols;
  return n > 0 && b.rows > 0 && b.cols > 0 && a.g_dtype == b.g_dtype && follows(a.G, b.G, n, bytes_of(a.g_dtype)) && dense(a, out) && dense(b, out) &&
         (!out || (a.out_dtype == b.out_dtype && follows(a.out, b.out, n, bytes_of(a.out_dtype))));
}
bool dense(const dion_param& a, bool v) {
  return a.rows == 1 || (a.ldx == a.cols && a.ldg == a.cols && a.ldm == a.cols && (!v || a.ldv == a.cols) && (a.X16 == nullptr || a.ldx16 == a.cols));
}
bool continues(const dion_param& a, const dion_param& b, bool v) {
  const i64 n = a.rows * a.cols;
  return n > 0 && b.rows > 0 && b.cols > 0 && follows(a.X, b.X, n, 4) && a.g_dtype == b.g_dtype && follows(a.G, b.G, n, bytes_of(a.g_dtype)) &&
         a.m_dtype == b.m_dtype && follows(a.M, b.M, n, bytes_of(a.m_dtype)) && (!v || follows(a.V, b.V, n, 4)) &&
         (a.X16 == nullptr ? b.X16 == nullptr : follows(a.X16, b.X16, n, 2)) && a.lr_scale == b.lr_scale && a.weight_decay == b.weight_decay &&
         dense(a, v) && dense(b, v);
}
// The array at list[*at] with all that continue it, as one; *at is then behind them.
template <class D>
void take(const D* list, int count, bool more, int* at, i64* rows, i64* cols) {
  int i = *at;
  *rows = list[i].rows; *cols = list[i].cols;
  for (; i + 1 < count && continues(list[i], list[i + 1], more); ++i) {
    *cols = *rows * *cols + list[i + 1].rows * list[i + 1].cols;
    *rows = 1;
  }
  *at = i + 1;
}

// Calls f on the smallest table that holds the items of a filled one.
template <int CAP, class Item, int BIG>
void shrink(const Table<Item, BIG>& from, Table<Item, CAP>* to) {
  to->tiles = from.tiles;
  to->count = from.count;
  std::copy(from.item, from.item + from.count, to->item);
}
template <class Item, int BIG, class F>
int by_count(Table<Item, BIG>& t, const F& f) {
  if (t.count <= FEW) { Table<Item, FEW> s; shrink(t, &s); return f(s); }
  if (t.count <= SOME) { Table<Item, SOME> s; shrink(t, &s); return f(s); }
  if (t.count <= MORE) { Table<Item, MORE> s; shrink(t, &s); return f(s); }
  return f(t);
}

void put(const dion_grad* list, int count, bool apart, int* done, Table<NormItem, MANY_NORM>* t) {
  const dion_grad& a = list[*done];
  NormItem* it = &t->item[t->count++];
  i64 rows = a.rows, cols = a.cols;
  if (apart) ++*done; else take(list, count, false, done, &rows, &cols);
  it->g = a.G; it->ldg = a.ldg;
  const Array arrays[] = {{a.G, a.ldg, shift_of(a.g_dtype)}};
  it->w = plan(rows, cols, a.g_dtype, DION_F32, arrays, &t->tiles);
}

// `left`: asks for the blocks' sums to be left as they are, for the launch behind, every block of which adds them up (clipping 262144
// elements 5.7 -> 4.9 us, 4.2M 9.5 -> 8.8, 33.6M 55.1 -> 54.7); how many, or 0 where they were added up after all (a list of several
// launches, or one whose scaling has many blocks).
int norm_launches(const Where& w, const dion_grad* list, int count, bool inf, NormOut o, float* each, int* left = nullptr) {
  Table<NormItem, MANY_NORM> t;
  int done = 0;
  if (left != nullptr) *left = 0;
  do {
    t.tiles = 0;
    t.count = 0;
    o.each = each != nullptr ? each + done : nullptr;
    o.use_carry = done > 0;
    while (done < count && t.count < MANY_NORM) put(list, count, each != nullptr, &done, &t);
    o.last = done == count;
    o.leave = left != nullptr && o.last && !o.use_carry && t.tiles / SCALE_SHAPE.tiles_one_wave <= (i64)w.sm_count * SCALE_SHAPE.resident;
    if (o.leave) *left = (int)blocks_for(w, NORM_SHAPE, t.tiles);
    LIST_TRY(by_count(t, [&](auto& table) {
      constexpr int CAP = sizeof(table.item) / sizeof(NormItem);
      return inf ? launch(w, k_list_norm<CAP, true>, NORM_SHAPE, table, o) : launch(w, k_list_norm<CAP, false>, NORM_SHAPE, table, o);
    }));
  } while (done < count);
  return DION_OK;
}

// `scale` false: the norm alone is wanted, `out` is not looked at.
template <int CAP>
void put(const dion_grad* list, int count, bool scale, int* done, Table<ScaleItem, CAP>* t) {
  const dion_grad& a = list[*done];
  ScaleItem* it = &t->item[t->count++];
  i64 rows, cols;
  take(list, count, scale, done, &rows, &cols);
  it->g = a.G; it->ldg = a.ldg;
  it->out = a.out; it->ldo = a.ldo;
  const Array arrays[] = {{a.G, a.ldg, shift_of(a.g_dtype)}, {scale ? a.out : nullptr, a.ldo, shift_of(a.out_dtype)}};
  it->w = plan(rows, cols, a.g_dtype, a.out_dtype, arrays, &t->tiles);
}

int scale_launches(const Where& w, const dion_grad* list, int count, Clip c) {
  Table<ScaleItem, MANY_SCALE> t;
  int done = 0;
  do {
    t.tiles = 0;
    t.count = 0;
    c.in_place = 1;
    while (done < count && t.count < MANY_SCALE) {
      c.in_place = c.in_place && list[done].G == list[done].out;
      put(list, count, true, &done, &t);
    }
    LIST_TRY(by_count(t, [&](auto& table) { return launch(w, k_list_scale<sizeof(table.item) / sizeof(ScaleItem)>, SCALE_SHAPE, table, c); }));
    c.norm_out = nullptr; c.coef_out = nullptr;
  } while (done < count);
  return DION_OK;
}

// A short list in one launch (k_list_cluster).  false: it is too long.
template <int CAP>
int cluster_launch(const Where& w, Table<ScaleItem, CAP>& t, bool scale, bool inf, const NormOut& o) {
  t.per = t.tiles / CLUSTER; t.rem = t.tiles % CLUSTER;
  return inf ? launch_blocks(w, k_list_cluster<CAP, true>, CLUSTER, THREADS * TEAMS, CLUSTER, t, o, (int)scale)
             : launch_blocks(w, k_list_cluster<CAP, false>, CLUSTER, THREADS * TEAMS, CLUSTER, t, o, (int)scale);
}
bool one_launch(const Where& w, const dion_grad* list, int count, bool scale, bool inf, const NormOut& o, int* rc) {
  Table<ScaleItem, MANY_CLUSTER> t;
  t.tiles = 0;
  t.count = 0;
  for (int done = 0; done < count;) {
    if (t.count == MANY_CLUSTER) return false;
    put(list, count, scale, &done, &t);
    if (t.tiles > CLUSTER_TILES) return false;
  }
  if (t.count <= FEW) {
    Table<ScaleItem, FEW> s;
    shrink(t, &s);
    *rc = cluster_launch(w, s, scale, inf, o);
  } else {
    *rc = cluster_launch(w, t, scale, inf, o);
  }
  return true;
}

template <bool ADAMW>
int step(const Where& w, const dion_param* list, int count, Rule r, float lr) {
  Table<StepItem, MANY_STEP> t;
  int done = 0;
  while (done < count) {
    t.tiles = 0;
    t.count = 0;
    r.first = done == 0;
    while (done < count && t.count < MANY_STEP) {
      const dion_param& a = list[done];
      StepItem* it = &t.item[t.count++];
      i64 rows, cols;
      take(list, count, ADAMW, &done, &rows, &cols);
      it->X = (float*)a.X; it->ldx = a.ldx;
      it->G = a.G; it->ldg = a.ldg;
      it->M = a.M; it->ldm = a.ldm;
      it->V = ADAMW ? (float*)a.V : nullptr; it->ldv = a.ldv;
      it->X16 = (__nv_bfloat16*)a.X16; it->ldx16 = a.ldx16;
      it->lr = lr * a.lr_scale;
      it->keep = (float)(1.0 - (double)lr * a.lr_scale * a.weight_decay);
      const Array arrays[] = {{a.G, a.ldg, shift_of(a.g_dtype)}, {it->X, a.ldx, 2}, {a.M, a.ldm, shift_of(a.m_dtype)}, {it->V, a.ldv, 2}, {it->X16, a.ldx16, 1}};
      it->w = plan(rows, cols, a.g_dtype, a.m_dtype, arrays, &t.tiles);
    }
    LIST_TRY(by_count(t, [&](auto& table) {
      constexpr int CAP = sizeof(table.item) / sizeof(StepItem);
      return launch(w, k_list_step<CAP, ADAMW>, ADAMW ? ADAMW_SHAPE : LION_SHAPE, table, r);
    }));
  }
  return DION_OK;
}

template <typename K>
bool load(K kernel) {
  cudaFuncAttributes fa;
  if (cudaFuncGetAttributes(&fa, kernel) != cudaSuccess) { cudaGetLastError(); return false; }
  return true;
}

}  // namespace

size_t scratch_bytes() { return (sizeof(Scratch) + 127) / 128 * 128; }
static_assert(MANY_NORM <= MOST_ARRAYS, "a launch's partial results fit");

namespace {

template <int CAP>
bool load_tables() {
  return load(k_list_norm<CAP, false>) && load(k_list_norm<CAP, true>) && load(k_list_scale<CAP>) && load(k_list_step<CAP, false>) &&
         load(k_list_step<CAP, true>);
}

}  // namespace

int configure() {
  const bool ok = load_tables<FEW>() && load_tables<SOME>() && load_tables<MORE>() && load(k_list_norm<MANY_NORM, false>) &&
                  load(k_list_norm<MANY_NORM, true>) && load(k_list_scale<MANY_SCALE>) && load(k_list_step<MANY_STEP, false>) &&
                  load(k_list_step<MANY_STEP, true>) && load(k_list_cluster<FEW, false>) && load(k_list_cluster<FEW, true>) &&
                  load(k_list_cluster<MANY_CLUSTER, false>) && load(k_list_cluster<MANY_CLUSTER, true>);
  return ok ? DION_OK : DION_ERR_CUDA;
}

int check_norm(const dion_grad* list, int count, int norm_type, float max_norm, const float* norm_out, const float* each_out, const float* coef_out) {
  if (count < 0 || (count > 0 && list == nullptr) || !norm_type_ok(norm_type)) return DION_ERR_INVALID;
  if (norm_out == nullptr && each_out == nullptr && coef_out == nullptr) return DION_ERR_INVALID;
  if (coef_out != nullptr && !(max_norm >= 0.f)) return DION_ERR_INVALID;
  LIST_TRY(check_floats(norm_out));
  LIST_TRY(check_floats(each_out));
  LIST_TRY(check_floats(coef_out));
  for (int i = 0; i < count; ++i) {
    const dion_grad& a = list[i];
    if (!known_type(a.g_dtype)) return DION_ERR_INVALID;
    LIST_TRY(check_shape(a.rows, a.cols));
    LIST_TRY(check_array(a.G, a.rows, a.cols, a.ldg, bytes_of(a.g_dtype)));
  }
  // the outputs against one another and against every array (the arrays are only read)
  const Range out[] = {range_of(norm_out, 1, norm_out != nullptr, 1, 4, true), range_of(each_out, 1, each_out != nullptr ? count : 0, count, 4, true),
                       range_of(coef_out, 1, coef_out != nullptr, 1, 4, true)};
  for (int k = 0; k < 3; ++k) {
    for (int j = k + 1; j < 3; ++j)
      if (conflict(out[k], out[j])) return DION_ERR_ALIAS;
    for (int i = 0; i < count; ++i)
      if (list[i].rows > 0 && list[i].cols > 0 && conflict(out[k], range_of(list[i].G, list[i].rows, list[i].cols, list[i].ldg, bytes_of(list[i].g_dtype), false)))
        return DION_ERR_ALIAS;
  }
  return DION_OK;
}

int check_clip(const dion_grad* list, int count, float max_norm, int norm_type, const float* norms, int num_norms,
               const float* norm_out, const float* coef_out) {
  if (count < 0 || (count > 0 && list == nullptr) || !norm_type_ok(norm_type) || !(max_norm >= 0.f)) return DION_ERR_INVALID;
  if ((norms == nullptr) != (num_norms == 0) || num_norms < 0) return DION_ERR_INVALID;
  LIST_TRY(check_floats(norms));
  LIST_TRY(check_floats(norm_out));
  LIST_TRY(check_floats(coef_out));
  const auto in_place = [](const dion_grad& a) { return a.G == a.out && a.g_dtype == a.out_dtype && (a.ldg == a.ldo || a.rows <= 1); };
  Runs kind[5];
  for (int i = 0; i < count; ++i) {
    const dion_grad& a = list[i];
    if (!known_type(a.g_dtype) || !known_type(a.out_dtype)) return DION_ERR_INVALID;
    LIST_TRY(check_shape(a.rows, a.cols));
    LIST_TRY(check_array(a.G, a.rows, a.cols, a.ldg, bytes_of(a.g_dtype)));
    LIST_TRY(check_array(a.out, a.rows, a.cols, a.ldo, bytes_of(a.out_dtype)));
    if (!in_place(a)) kind[0].add(a.G, a.rows, a.cols, a.ldg, bytes_of(a.g_dtype));
    kind[1].add(a.out, a.rows, a.cols, a.ldo, bytes_of(a.out_dtype));
  }
  kind[2].add(norms, 1, num_norms, num_norms, 4);
  kind[3].add(norm_out, 1, 1, 1, 4);
  kind[4].add(coef_out, 1, 1, 1, 4);
  return check_ranges(kind, [&](auto range) {
    for (int i = 0; i < count; ++i) {
      const dion_grad& a = list[i];
      if (!in_place(a)) range(a.G, a.rows, a.cols, a.ldg, bytes_of(a.g_dtype), false);
    }
    for (int i = 0; i < count; ++i) range(list[i].out, list[i].rows, list[i].cols, list[i].ldo, bytes_of(list[i].out_dtype), true);
    range(norms, 1, num_norms, num_norms, 4, false);
    range(norm_out, 1, 1, 1, 4, true);
    range(coef_out, 1, 1, 1, 4, true);
  });
}

int check_step(bool adamw, const dion_param* list, int count, const dion_rule* rule, float lr) {
  if (count < 0 || (count > 0 && list == nullptr) || rule == nullptr || !isfinite(lr)) return DION_ERR_INVALID;
  if (!(rule->beta1 >= 0.0 && rule->beta1 < 1.0) || !(rule->beta2 >= 0.0 && rule->beta2 < 1.0)) return DION_ERR_INVALID;
  // (the step's quotient is within its bound for divisors in this range; below it V's root alone is never, but zero)
  if (adamw && rule->eps != 0.0 && !(rule->eps >= 0x1p-126 && rule->eps <= 0x1p125)) return DION_ERR_INVALID;
  if (adamw && rule->step_dev == nullptr && rule->step < 1) return DION_ERR_INVALID;
  if ((uintptr_t)rule->step_dev & 7) return DION_ERR_ALIGN;
  LIST_TRY(check_floats(rule->grad_scale));
  Runs kind[7];
  for (int i = 0; i < count; ++i) {
    const dion_param& a = list[i];
    if (!known_type(a.g_dtype) || !known_type(a.m_dtype) || !isfinite(a.lr_scale) || !isfinite(a.weight_decay)) return DION_ERR_INVALID;
    LIST_TRY(check_shape(a.rows, a.cols));
    LIST_TRY(check_array(a.X, a.rows, a.cols, a.ldx, 4));
    LIST_TRY(check_array(a.G, a.rows, a.cols, a.ldg, bytes_of(a.g_dtype)));
    LIST_TRY(check_array(a.M, a.rows, a.cols, a.ldm, bytes_of(a.m_dtype)));
    if (adamw) LIST_TRY(check_array(a.V, a.rows, a.cols, a.ldv, 4));
    if (a.X16 != nullptr) LIST_TRY(check_array(a.X16, a.rows, a.cols, a.ldx16, 2));
    kind[0].add(a.X, a.rows, a.cols, a.ldx, 4);
    kind[1].add(a.G, a.rows, a.cols, a.ldg, bytes_of(a.g_dtype));
    kind[2].add(a.M, a.rows, a.cols, a.ldm, bytes_of(a.m_dtype));
    if (adamw) kind[3].add(a.V, a.rows, a.cols, a.ldv, 4);
    kind[4].add(a.X16, a.rows, a.cols, a.ldx16, 2);
  }
  if (adamw) kind[5].add(rule->step_dev, 1, 1, 1, 8);
  kind[6].add(rule->grad_scale, 1, 1, 1, 4);
  return check_ranges(kind, [&](auto range) {
    for (int i = 0; i < count; ++i) range(list[i].X, list[i].rows, list[i].cols, list[i].ldx, 4, true);
    for (int i = 0; i < count; ++i) range(list[i].G, list[i].rows, list[i].cols, list[i].ldg, bytes_of(list[i].g_dtype), false);
    for (int i = 0; i < count; ++i) range(list[i].M, list[i].rows, list[i].cols, list[i].ldm, bytes_of(list[i].m_dtype), true);
    for (int i = 0; i < count && adamw; ++i) range(list[i].V, list[i].rows, list[i].cols, list[i].ldv, 4, true);
    for (int i = 0; i < count; ++i) range(list[i].X16, list[i].rows, list[i].cols, list[i].ldx16, 2, true);
    if (adamw) range(rule->step_dev, 1, 1, 1, 8, false);
    range(rule->grad_scale, 1, 1, 1, 4, false);
  });
}

namespace {

NormOut norm_out_of(const Where& w, float max_norm, float* norm_out, float* coef_out) {
  NormOut o = {};
  o.norm = norm_out; o.coef = coef_out; o.max_norm = max_norm;
  o.status = w.status;
  return o;
}

// hi is the largest float below beta, lo the rest.
Beta split(double beta) {
  float hi = (float)beta;
  if (hi > 0.f && (double)hi >= beta) hi = nextafterf(hi, 0.f);
  return {hi, (float)(beta - (double)hi)};
}

}  // namespace

int grad_norm(const Where& w, const dion_grad* list, int count, int norm_type, float max_norm, float* norm_out, float* each_out,
              float* coef_out) {
  NormOut o = norm_out_of(w, max_norm, norm_out, coef_out);
  const bool inf = norm_type == DION_NORM_INF;
  int rc;
  if (each_out == nullptr && one_launch(w, list, count, false, inf, o, &rc)) return rc;
  o.scratch = (Scratch*)w.scratch(w.owner, w.stream);
  return norm_launches(w, list, count, inf, o, each_out);
}

int clip_grads(const Where& w, const dion_grad* list, int count, float max_norm, int norm_type, const float* norms, int num_norms,
               float* norm_out, float* coef_out) {
  Clip c = {};
  c.max_norm = max_norm; c.inf = norm_type == DION_NORM_INF;
  c.status = w.status;
  if (norms != nullptr) {
    c.norms = norms; c.count = num_norms; c.norm_out = norm_out; c.coef_out = coef_out;
  } else {
    NormOut o = norm_out_of(w, max_norm, norm_out, coef_out);
    int rc;
    if (one_launch(w, list, count, true, c.inf, o, &rc)) return rc;
    o.scratch = (Scratch*)w.scratch(w.owner, w.stream);
    int left;
    LIST_TRY(norm_launches(w, list, count, c.inf, o, nullptr, &left));
    if (left > 0) {
      c.sums = o.scratch->part; c.count = left; c.norm_out = norm_out; c.coef_out = coef_out;
    } else {
      c.coef = &o.scratch->coef;
    }
  }
  return scale_launches(w, list, count, c);
}

int param_step(const Where& w, bool adamw, const dion_param* list, int count, const dion_rule* rule, float lr) {
  Rule r = {};
  r.beta1 = rule->beta1; r.beta2 = rule->beta2;
  r.b1 = (float)rule->beta1; r.c1 = (float)(1.0 - rule->beta1);
  const double of_m = adamw ? rule->beta1 : rule->beta2;
  r.m = split(of_m); r.cm = (float)(1.0 - of_m);
  r.v = split(rule->beta2); r.cv = (float)(1.0 - rule->beta2);
  r.eps = (float)rule->eps;
  r.step_dev = adamw ? rule->step_dev : nullptr;
  if (adamw && rule->step_dev == nullptr) {
    r.inv1 = (float)(1.0 / (1.0 - pow(rule->beta1, (double)rule->step)));
    r.inv2 = (float)(1.0 / (1.0 - pow(rule->beta2, (double)rule->step)));
  }
  r.scale = rule->grad_scale;
  r.status = w.status;
  return adamw ? step<true>(w, list, count, r, lr) : step<false>(w, list, count, r, lr);
}

}  // namespace list
}  // namespace dion
