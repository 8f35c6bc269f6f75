// Rotary positions on their own, and the paged KV cache: rows written (rotated and quantised on the way) and
// read back (sm_103a).
//
// All three move each element once and do a few operations on it, so HBM is what bounds them.  A thread takes
// 16 elements of one head, in 16-byte pieces of its input or output that lie beside its neighbours' pieces (two pieces
// of one lane side by side would fill each 32-byte sector in two stores).  In the half layout element j of a head is
// turned together with element j + rot_dim / 2: the pieces are chosen to hold each other's partners, so no
// value crosses threads before it is stored, and rows may be rotated in place.  The cosines and sines of a row
// are shared by all its heads: a CTA takes a few rows with all their heads and computes each angle once, into
// shared memory, while its first loads are on their way.
//
// Measured (device time, of the measured copy rate): q and k of 23,819 rows, 64 heads x 128 in fp16, rotated in 115 us (100%);
// 8,129 rows of 32 heads in fp32 40 us (97%); 17,858 rows of 32 heads written as e4m3 80 us (81%: 57% of the issue slots,
// about 200 instructions for the 512 elements of a warp) and read back in 69 us (93%).  Two items a thread at a time: with
// four the registers leave too few CTAs (rope 153 us for 123 at that step); pieces of one lane side by side 70 us where
// a sequence is read back in 60.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kv_pages.cuh"
#include "rift_internal.h"
#include "rope_angle.cuh"

namespace rift {

__device__ unsigned int g_err_kv;

unsigned int read_clear_err_kv() {
  unsigned int v = 0, z = 0;
  cudaMemcpyFromSymbol(&v, g_err_kv, sizeof(v));
  cudaMemcpyToSymbol(g_err_kv, &z, sizeof(z));
  return v;
}

namespace {

constexpr int KV_THREADS = 256;
constexpr int TABLE = 2048;   // (cos, sin) pairs a CTA holds: 16 KB
constexpr int MAX_ROWS = 64;  // rows of a CTA
constexpr int U = 2;          // items (16 elements) whose loads a thread issues together

// n / d and n % d for 0 <= n < 2^31 by a multiplication: with m = ceil(2^32 / d), n m / 2^32 is n / d or one more.
struct Divider {
  uint32_t d, m;
  __device__ __forceinline__ void operator()(uint32_t n, uint32_t& q, uint32_t& r) const {
    q = d == 1 ? n : __umulhi(n, m);
    r = n - q * d;
    if ((int)r < 0) {
      --q;
      r += d;
    }
  }
};
Divider divider(uint32_t d) { return {d, (uint32_t)((0x100000000ull + d - 1) / d)}; }

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// The elements of a head that lane i of its head_dim / 16 lanes takes: four groups of 4, as (x0, x1) and (y0, y1).
// PIECE 8: x1 and y1 follow x0 and y0; PIECE 4: each group is a piece of its own.  In the half layout the
// first rot_dim / 16 lanes take the turned elements, x in the first half and y its partners in the
// second; the others, and all in the interleaved layout (rot_dim 0 here), split what is left evenly.
struct Spots {
  int x0, x1, y0, y1;
};
template <int PIECE>
__device__ __forceinline__ Spots spots_of(int i, int lanes, int rot_dim) {
  const int n = rot_dim / 16;
  if (i < n) {
    if (PIECE == 8) return {8 * i, 8 * i + 4, 8 * i + rot_dim / 2, 8 * i + rot_dim / 2 + 4};
    return {4 * i, 4 * (i + n), 4 * i + rot_dim / 2, 4 * (i + n) + rot_dim / 2};
  }
  const int m = lanes - n, k = i - n;
  if (PIECE == 8) return {rot_dim + 8 * k, rot_dim + 8 * k + 4, rot_dim + 8 * (k + m), rot_dim + 8 * (k + m) + 4};
  return {rot_dim + 4 * k, rot_dim + 4 * (k + m), rot_dim + 4 * (k + 2 * m), rot_dim + 4 * (k + 3 * m)};
}
template <typename T>
constexpr int PIECE = 16 / sizeof(T);

// A lane's 16 elements as they lie in memory, in pieces of N.
template <typename T, int N>
struct Raw;
template <typename T>
struct Raw<T, 8> {  // 16-bit elements
  uint4 x, y;
  __device__ __forceinline__ void load(const T* p, Spots s) {
    x = *reinterpret_cast<const uint4*>(p + s.x0);
    y = *reinterpret_cast<const uint4*>(p + s.y0);
  }
};
template <typename T>
struct Raw<T, 4> {  // 16-bit elements, in pieces of four
  uint2 x0, x1, y0, y1;
  __device__ __forceinline__ void load(const T* p, Spots s) {
    x0 = *reinterpret_cast<const uint2*>(p + s.x0);
    x1 = *reinterpret_cast<const uint2*>(p + s.x1);
    y0 = *reinterpret_cast<const uint2*>(p + s.y0);
    y1 = *reinterpret_cast<const uint2*>(p + s.y1);
  }
};
template <>
struct Raw<float, 4> {
  float4 x0, x1, y0, y1;
  __device__ __forceinline__ void load(const float* p, Spots s) {
    x0 = *reinterpret_cast<const float4*>(p + s.x0);
    x1 = *reinterpret_cast<const float4*>(p + s.x1);
    y0 = *reinterpret_cast<const float4*>(p + s.y0);
    y1 = *reinterpret_cast<const float4*>(p + s.y1);
  }
};
template <>
struct Raw<e4m3_t, 8> {
  uint2 x, y;
  __device__ __forceinline__ void load(const e4m3_t* p, Spots s) {
    x = *reinterpret_cast<const uint2*>(p + s.x0);
    y = *reinterpret_cast<const uint2*>(p + s.y0);
  }
};
template <>
struct Raw<e4m3_t, 4> {
  uint32_t x0, x1, y0, y1;
  __device__ __forceinline__ void load(const e4m3_t* p, Spots s) {
    x0 = *reinterpret_cast<const uint32_t*>(p + s.x0);
    x1 = *reinterpret_cast<const uint32_t*>(p + s.x1);
    y0 = *reinterpret_cast<const uint32_t*>(p + s.y0);
    y1 = *reinterpret_cast<const uint32_t*>(p + s.y1);
  }
};

__device__ __forceinline__ void pair_f32(uint32_t w, float* f, __half) {
  const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w));
  f[0] = t.x;
  f[1] = t.y;
}
__device__ __forceinline__ void pair_f32(uint32_t w, float* f, __nv_bfloat16) {
  f[0] = __uint_as_float(w << 16);
  f[1] = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void four_f32(uint32_t w, float* f) {
  uint32_t lo, hi;
  half2s_of(w, lo, hi);
  pair_f32(lo, f, __half());
  pair_f32(hi, f + 2, __half());
}
template <typename T>
__device__ __forceinline__ void values(const Raw<T, 8>& r, float (&a)[8], float (&b)[8]) {
  const uint32_t x[4] = {r.x.x, r.x.y, r.x.z, r.x.w}, y[4] = {r.y.x, r.y.y, r.y.z, r.y.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    pair_f32(x[e], a + 2 * e, T());
    pair_f32(y[e], b + 2 * e, T());
  }
}
template <typename T>
__device__ __forceinline__ void values(const Raw<T, 4>& r, float (&a)[8], float (&b)[8]) {
  pair_f32(r.x0.x, a, T());
  pair_f32(r.x0.y, a + 2, T());
  pair_f32(r.x1.x, a + 4, T());
  pair_f32(r.x1.y, a + 6, T());
  pair_f32(r.y0.x, b, T());
  pair_f32(r.y0.y, b + 2, T());
  pair_f32(r.y1.x, b + 4, T());
  pair_f32(r.y1.y, b + 6, T());
}
__device__ __forceinline__ void values(const Raw<float, 4>& r, float (&a)[8], float (&b)[8]) {
  const float4 v[4] = {r.x0, r.x1, r.y0, r.y1};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float* f = (k < 2 ? a : b) + 4 * (k & 1);
    f[0] = v[k].x;
    f[1] = v[k].y;
    f[2] = v[k].z;
    f[3] = v[k].w;
  }
}
__device__ __forceinline__ void values(const Raw<e4m3_t, 8>& r, float (&a)[8], float (&b)[8]) {
  four_f32(r.x.x, a);
  four_f32(r.x.y, a + 4);
  four_f32(r.y.x, b);
  four_f32(r.y.y, b + 4);
}
__device__ __forceinline__ void values(const Raw<e4m3_t, 4>& r, float (&a)[8], float (&b)[8]) {
  four_f32(r.x0, a);
  four_f32(r.x1, a + 4);
  four_f32(r.y0, b);
  four_f32(r.y1, b + 4);
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi, __half) { return pack_half2(lo, hi); }
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __nv_bfloat16) { return pack_bf16x2(lo, hi); }
// 8 values into two groups of 4 elements.
template <typename T>
__device__ __forceinline__ void store8(T* p, int s0, int s1, const float (&f)[8]) {
  const uint2 a = make_uint2(pack2(f[0], f[1], T()), pack2(f[2], f[3], T())),
              b = make_uint2(pack2(f[4], f[5], T()), pack2(f[6], f[7], T()));
  if (s1 == s0 + 4 && s0 % 8 == 0) {
    *reinterpret_cast<uint4*>(p + s0) = make_uint4(a.x, a.y, b.x, b.y);
  } else {
    *reinterpret_cast<uint2*>(p + s0) = a;
    *reinterpret_cast<uint2*>(p + s1) = b;
  }
}
__device__ __forceinline__ void store8(float* p, int s0, int s1, const float (&f)[8]) {
  *reinterpret_cast<float4*>(p + s0) = make_float4(f[0], f[1], f[2], f[3]);
  *reinterpret_cast<float4*>(p + s1) = make_float4(f[4], f[5], f[6], f[7]);
}

// (a, b) turned: each product and each sum a rounded fp32 operation.
__device__ __forceinline__ void turn(float& a, float& b, float2 cs) {
  const float x = __fsub_rn(__fmul_rn(a, cs.x), __fmul_rn(b, cs.y));
  b = __fadd_rn(__fmul_rn(b, cs.x), __fmul_rn(a, cs.y));
  a = x;
}

// The (cos, sin) of nr rows' pairs, where `at` puts them (row, pair).  The frequencies come from `turns`, a copy in shared
// memory: lanes that read different entries of a kernel's arguments wait for each other.  From the arguments and so, us:
// a million rows of one head of 64, 278 and 211, of one head of 128, 549 and 393.
template <typename Pos, typename At>
__device__ __forceinline__ void fill_table(float2* table, const uint64_t* turns, const RopeAngles& R, int nr, Divider half,
                                           Pos pos, At at) {
  for (uint32_t t = threadIdx.x; t < nr * half.d; t += KV_THREADS) {
    uint32_t r, j;
    half(t, r, j);
    float2 v = cos_sin_of_turns((uint64_t)(long long)pos(r) * turns[j], {R.amplitude, R.amplitude_rest});
    if (R.inverse) v.y = -v.y;
    table[at(r, j)] = v;
  }
}

// A row's table holds pair j at (j % 4) * ceil(half / 4) + j / 4: the lanes of a head, whose groups of four follow
// each other, read entries that do so too.
__device__ __forceinline__ int table_at(int j, int quarter) { return (j & 3) * quarter + (j >> 2); }

// A lane's elements turned by the row's table (half layout: rot_dim a multiple of 16).
__device__ __forceinline__ void turn_spots(float (&a)[8], float (&b)[8], Spots s, const float2* table, int half,
                                           bool interleaved) {
  const int quarter = (half + 3) / 4;
  if (!interleaved) {
    if (s.x0 >= half) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      turn(a[e], b[e], table[e * quarter + (s.x0 >> 2)]);
      turn(a[4 + e], b[4 + e], table[e * quarter + (s.x1 >> 2)]);
    }
    return;
  }
  const int at[4] = {s.x0 / 2, s.x1 / 2, s.y0 / 2, s.y1 / 2};  // the first pair of each group
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float* f = (k < 2 ? a : b) + 4 * (k & 1) + 2 * e;
      if (at[k] + e < half) turn(f[0], f[1], table[table_at(at[k] + e, quarter)]);
    }
}

// ------------------------------------------------------------------------------------------ rope

// `rows` rows of x a CTA, with all their heads (gridDim.y CTAs share them where there are few rows).  16-byte aligned
// rows of heads of a multiple of 16 elements.
template <typename T>
__global__ void __launch_bounds__(KV_THREADS) rope_kernel(const T* x, int n_rows, int head_dim, int x_stride,
                                                          const int* __restrict__ positions,
                                                          const __grid_constant__ RopeAngles R, T* out, int out_stride,
                                                          int rows, Divider per_row, Divider lanes, Divider by_half) {
  __shared__ float2 table[TABLE];
  __shared__ uint64_t turns[RIFT_ROPE_MAX_HEAD_DIM / 2];
  if (threadIdx.x < R.rot_dim / 2) turns[threadIdx.x] = R.turns[threadIdx.x];
  pdl_trigger();
  pdl_wait();
  const int half = R.rot_dim / 2, quarter = (half + 3) / 4;
  const int r0 = blockIdx.x * rows, nr = min(rows, n_rows - r0), items = nr * (int)per_row.d;
  const T* x0 = x + (long long)r0 * x_stride;
  T* out0 = out + (long long)r0 * out_stride;
  Raw<T, PIECE<T>> raw[U];
  uint32_t r[U], h[U];
  Spots s[U];
  auto load = [&](int t0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * KV_THREADS;
      if (t >= items) break;
      uint32_t col, i;
      per_row(t, r[u], col);
      lanes(col, h[u], i);
      s[u] = spots_of<PIECE<T>>(i, lanes.d, R.interleaved ? 0 : R.rot_dim);
      raw[u].load(x0 + (long long)r[u] * x_stride + h[u] * head_dim, s[u]);
    }
  };
  int t0 = blockIdx.y * U * KV_THREADS + threadIdx.x;
  load(t0);
  __syncthreads();
  fill_table(table, turns, R, nr, by_half, [&](int r) { return positions[r0 + r]; },
             [&](int r, int j) { return r * 4 * quarter + table_at(j, quarter); });
  __syncthreads();
  for (;;) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t0 + u * KV_THREADS >= items) break;
      float a[8], b[8];
      values(raw[u], a, b);
      turn_spots(a, b, s[u], table + r[u] * 4 * quarter, half, R.interleaved);
      T* o = out0 + (long long)r[u] * out_stride + h[u] * head_dim;
      store8(o, s[u].x0, s[u].x1, a);
      store8(o, s[u].y0, s[u].y1, b);
    }
    t0 += gridDim.y * U * KV_THREADS;
    if (t0 >= items) break;
    load(t0);
  }
}

// Any even head_dim, rot_dim and strides: a thread per pair of elements.
template <typename T>
__global__ void __launch_bounds__(KV_THREADS) rope_pairs_kernel(const T* x, int n_rows, int head_dim, int x_stride,
                                                                const int* __restrict__ positions,
                                                                const __grid_constant__ RopeAngles R, T* out,
                                                                int out_stride, int rows, Divider per_row,
                                                                Divider pairs, Divider by_half) {
  __shared__ float2 table[TABLE];
  __shared__ uint64_t turns[RIFT_ROPE_MAX_HEAD_DIM / 2];
  if (threadIdx.x < R.rot_dim / 2) turns[threadIdx.x] = R.turns[threadIdx.x];
  pdl_trigger();
  pdl_wait();
  const int half = R.rot_dim / 2;
  const int r0 = blockIdx.x * rows, nr = min(rows, n_rows - r0), items = nr * (int)per_row.d;
  __syncthreads();
  fill_table(table, turns, R, nr, by_half, [&](int r) { return positions[r0 + r]; }, [&](int r, int j) { return r * half + j; });
  __syncthreads();
  for (int t = blockIdx.y * KV_THREADS + threadIdx.x; t < items; t += gridDim.y * KV_THREADS) {
    uint32_t r, col, h, j;
    per_row(t, r, col);
    pairs(col, h, j);
    const bool turned = (int)j < half;
    const int e0 = turned && !R.interleaved ? j : 2 * j, e1 = turned && !R.interleaved ? j + half : 2 * j + 1;
    const T* p = x + (long long)(r0 + r) * x_stride + h * head_dim;
    float a = to_f32(p[e0]), b = to_f32(p[e1]);
    if (turned) turn(a, b, table[r * half + j]);
    T* o = out + (long long)(r0 + r) * out_stride + h * head_dim;
    o[e0] = from_f32<T>(a);
    o[e1] = from_f32<T>(b);
  }
}

// Rows of a CTA: 64 KB of them (16 elements an item, `size` bytes each), but not so many that the GPU has fewer than four
// CTAs an SM to work on at once, and no more rows than the table holds.  (The items of rope_pairs_kernel are pairs: its CTAs
// get an eighth of that.)  Half and twice as much, us: rope of 23,819 rows
// 115, 115, 118 (32 KB, 64 KB, 128 KB); in fp32 40, 43, 46 (64, 128, 256); e4m3 read back 61, 59, 62; stored and read back
// 157, 150, 148.
int rows_of_cta(int n_rows, int per_row, int half, int size) {
  const int most = std::min(MAX_ROWS, half > 0 ? TABLE / ((half + 3) / 4 * 4) : MAX_ROWS);
  return std::max(1, std::min({(64 << 10) / (16 * size) / per_row, n_rows / 608 + (n_rows % 608 != 0), most}));
}
unsigned row_ctas(int n_rows, int rows) { return (unsigned)(((long long)n_rows + rows - 1) / rows); }
// CTAs that share a row's items: one, unless there are too few rows for the GPU.
int ctas_of_row(int n_rows, int per_row, int each) {
  return n_rows >= 304 ? 1 : std::max(1, std::min((per_row + each - 1) / each, 608 / n_rows));
}

template <typename T>
bool launch_rope_t(const void* x, int n_rows, int n_heads, int head_dim, long long x_stride, const int* positions,
                   const RopeAngles& R, void* out, long long out_stride, cudaStream_t st) {
  const long long align = 16 / sizeof(T);
  const bool vec = head_dim % 16 == 0 && (R.interleaved || R.rot_dim % 16 == 0) && x_stride % align == 0 &&
                   out_stride % align == 0;
  const int lanes = vec ? head_dim / 16 : head_dim / 2, per_row = n_heads * lanes;
  const int rows = rows_of_cta(n_rows, per_row, R.rot_dim / 2, (int)sizeof(T));
  const dim3 grid(row_ctas(n_rows, rows), ctas_of_row(n_rows, per_row, vec ? U * KV_THREADS : KV_THREADS));
  auto go = [&](auto kernel) {
    return launch_ex(kernel, grid, dim3(KV_THREADS), 0, st, true, static_cast<const T*>(x), n_rows, head_dim, (int)x_stride,
                     positions, R, static_cast<T*>(out), (int)out_stride, rows, divider(per_row), divider(lanes),
                     divider(R.rot_dim / 2)) == cudaSuccess;
  };
  return vec ? go(rope_kernel<T>) : go(rope_pairs_kernel<T>);
}

// ------------------------------------------------------------------------------------ the paged cache

// Where a row of a call lies in the pools: its first head's elements and scale byte; and its position.
struct Place {
  long long at, scale_at;
  int pos, state;
};
enum { IN_POOL, NO_SEQUENCE, LOST };  // of Place::state; LOST: it cannot be addressed (the error flag is set)

// The last sequence i with cu[i] <= r (0 before the first), by a whole warp: a binary search's steps each wait for the
// last one's load, so 32 probes at a time.
__device__ __forceinline__ int sequence_of(int r, const int* __restrict__ cu, int n_seq) {
  int lo = 0, span = n_seq;
  while (span > 1) {
    const int step = (span + 31) / 32, at = (threadIdx.x & 31) * step;
    const uint32_t below = __ballot_sync(0xffffffffu, at < span && cu[lo + at] <= r);
    const int k = max(0, 31 - __clz(below)) * step;
    lo += k;
    span = min(step, span - k);
  }
  return lo;
}

// The places of rows r0 .. r0 + nr - 1, by the CTA's first warp.
__device__ __forceinline__ void find_places(Place* place, const KvPool& P, int r0, int nr, const int* __restrict__ cu,
                                            const int* __restrict__ start, int n_seq, const int* __restrict__ table,
                                            int max_pages) {
  if (threadIdx.x >= 32) return;
  int i0 = 0, i1 = 0, first = 0, last = 0;
  if (cu) {
    first = cu[0];
    last = cu[n_seq];
    i0 = sequence_of(r0, cu, n_seq);
    i1 = nr > 1 ? sequence_of(r0 + nr - 1, cu, n_seq) : i0;
  }
  for (int k = threadIdx.x; k < nr; k += 32) {
    const int r = r0 + k;
    int i = r, off = 0;
    if (cu) {
      if (r < first || r >= last) {
        place[k] = {0, 0, 0, NO_SEQUENCE};
        continue;
      }
      int lo = i0, hi = i1 + 1;
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (cu[mid] <= r) lo = mid;
        else hi = mid;
      }
      i = lo;
      off = r - cu[i];
    }
    const long long pos = (long long)start[i] + off;
    Place w = {0, 0, (int)pos, LOST};
    if (pos < 0 || pos >= ((long long)max_pages << P.ps_shift)) {
      atomicOr(&g_err_kv, RIFT_EBIT_CAPACITY);
    } else {
      const int page = table[(long long)i * max_pages + (pos >> P.ps_shift)], row = (int)pos & ((1 << P.ps_shift) - 1);
      if (page >= 0 && page < P.n_pages) w = {P.at(page, row, 0), P.scale_at(page, row, 0), (int)pos, IN_POOL};
      else atomicOr(&g_err_kv, RIFT_EBIT_BADID);
    }
    place[k] = w;
  }
}

// Stores a lane's elements of one head's row (shared by `lanes` neighbouring lanes) in a 16-bit pool.
template <typename CT>
__device__ __forceinline__ void keep(CT* pool, uint8_t*, long long at, long long, Spots s, float (&a)[8],
                                     float (&b)[8], int, bool, bool ok) {
  if (!ok) return;
  store8(pool + at, s.x0, s.x1, a);
  store8(pool + at, s.y0, s.y1, b);
}
// ... as e4m3 codes over the row's power of two.  Every lane of the warp takes part in the shuffles.
template <>
__device__ __forceinline__ void keep<e4m3_t>(e4m3_t* pool, uint8_t* scale, long long at, long long scale_at, Spots s,
                                             float (&a)[8], float (&b)[8], int lanes, bool lane0, bool ok) {
  auto over_lanes = [&](float x) {  // 4 or 8 of them
    if (lanes == 8) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 4));
    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
    return fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
  };
  float top = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = fmaxf(top, fmaxf(fabsf(a[e]), fabsf(b[e])));  // NaN left out
  top = over_lanes(top);
  if (__any_sync(0xffffffffu, isinf(top))) {  // infinities become NaN: the conversion would saturate them
    top = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (isinf(a[e])) a[e] = a[e] - a[e];
      if (isinf(b[e])) b[e] = b[e] - b[e];
      top = fmaxf(top, fmaxf(fabsf(a[e]), fabsf(b[e])));
    }
    top = over_lanes(top);
  }
  if (!ok) return;
  const int byte = e4m3_scale_byte(top);
  const float inv = inv_scale_of(byte);
  auto codes = [&](const float* f) { return e4m3x4_of(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv); };
  uint8_t* p = reinterpret_cast<uint8_t*>(pool) + at;
  const uint2 x = make_uint2(codes(a), codes(a + 4)), y = make_uint2(codes(b), codes(b + 4));
  if (s.x1 == s.x0 + 4 && s.x0 % 8 == 0) {
    *reinterpret_cast<uint2*>(p + s.x0) = x;
    *reinterpret_cast<uint2*>(p + s.y0) = y;
  } else {
    *reinterpret_cast<uint32_t*>(p + s.x0) = x.x;
    *reinterpret_cast<uint32_t*>(p + s.x1) = x.y;
    *reinterpret_cast<uint32_t*>(p + s.y0) = y.x;
    *reinterpret_cast<uint32_t*>(p + s.y1) = y.y;
  }
  if (lane0) scale[scale_at] = (uint8_t)byte;
}

// `rows` rows a CTA: the places and angles of its rows, then every head of them (queries, keys, values).
template <typename T, typename CT>
__global__ void __launch_bounds__(KV_THREADS)
    append_kernel(const __grid_constant__ KvPool P, const T* __restrict__ k, int k_stride,
                  const T* __restrict__ v, int v_stride, int n_rows, const int* __restrict__ cu,
                  const int* __restrict__ start, int n_seq, const int* __restrict__ page_table, int max_pages,
                  bool rotate, const __grid_constant__ RopeAngles R, const T* q, int q_stride, int n_q, T* q_out,
                  int q_out_stride, int rows, Divider per_row, Divider lanes, Divider by_half) {
  __shared__ float2 table[TABLE];
  __shared__ uint64_t turns[RIFT_ROPE_MAX_HEAD_DIM / 2];
  __shared__ Place place[MAX_ROWS];
  if (threadIdx.x < R.rot_dim / 2) turns[threadIdx.x] = R.turns[threadIdx.x];
  pdl_trigger();
  pdl_wait();
  const int half = rotate ? R.rot_dim / 2 : 0, quarter = (half + 3) / 4;
  const int r0 = blockIdx.x * rows, nr = min(rows, n_rows - r0), items = nr * (int)per_row.d;
  Raw<T, PIECE<T>> raw[U];
  uint32_t r[U], h[U], i[U];
  Spots s[U];
  const T *q0 = q + (long long)r0 * q_stride, *k0 = k + (long long)r0 * k_stride, *v0 = v + (long long)r0 * v_stride;
  T* q_out0 = q_out + (long long)r0 * q_out_stride;
  auto load = [&](int t0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = min(t0 + u * KV_THREADS, items - 1);  // the last lanes of a CTA take part in the shuffles
      uint32_t col;
      per_row(t, r[u], col);
      lanes(col, h[u], i[u]);
      const int hh = h[u];
      const bool is_q = hh < n_q, is_k = hh < n_q + P.n_kv, turned = rotate && is_k;
      s[u] = spots_of<PIECE<T>>(i[u], lanes.d, turned && !R.interleaved ? R.rot_dim : 0);
      const T* p = is_q ? q0 : is_k ? k0 : v0;
      const int stride = is_q ? q_stride : is_k ? k_stride : v_stride, head = is_q ? hh : is_k ? hh - n_q : hh - n_q - P.n_kv;
      raw[u].load(p + (long long)r[u] * stride + head * P.head_dim, s[u]);
    }
  };
  int t0 = blockIdx.y * U * KV_THREADS + threadIdx.x;
  load(t0);
  find_places(place, P, r0, nr, cu, start, n_seq, page_table, max_pages);
  __syncthreads();
  if (rotate) {
    fill_table(table, turns, R, nr, by_half, [&](int r) { return place[r].pos; },
               [&](int r, int j) { return r * 4 * quarter + table_at(j, quarter); });
    __syncthreads();
  }
  for (;;) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool mine = t0 + u * KV_THREADS < items;
      const Place w = place[r[u]];
      const int hh = h[u];
      const bool is_q = hh < n_q, is_k = !is_q && hh < n_q + P.n_kv;
      float a[8], b[8];
      values(raw[u], a, b);
      if (rotate && (is_q || is_k)) {
        turn_spots(a, b, s[u], table + r[u] * 4 * quarter, half, R.interleaved);
        if (is_q) {
          if (mine && w.state != NO_SEQUENCE) {
            T* o = q_out0 + (long long)r[u] * q_out_stride + hh * P.head_dim;
            store8(o, s[u].x0, s[u].x1, a);
            store8(o, s[u].y0, s[u].y1, b);
          }
        } else {  // the turned key in the input's type, as a rotation on its own would leave it
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            a[e] = to_f32(from_f32<T>(a[e]));
            b[e] = to_f32(from_f32<T>(b[e]));
          }
        }
      }
      const bool held = mine && !is_q && w.state == IN_POOL;
      const int kvh = is_k ? hh - n_q : hh - n_q - P.n_kv;
      keep<CT>(static_cast<CT*>(is_k ? P.k : P.v), is_k ? P.k_scale : P.v_scale, w.at + (long long)kvh * P.head_stride,
               w.scale_at + (kvh << P.ps_shift), s[u], a, b, lanes.d, i[u] == 0, held);
    }
    t0 += gridDim.y * U * KV_THREADS;
    if (t0 - (int)threadIdx.x >= items) break;  // whole CTAs: the lanes of a head exchange their maxima
    load(t0);
  }
}

template <typename T, typename CT>
__global__ void __launch_bounds__(KV_THREADS)
    gather_kernel(const __grid_constant__ KvPool P, int n_rows, const int* __restrict__ cu,
                  const int* __restrict__ start, int n_seq, const int* __restrict__ page_table, int max_pages,
                  T* __restrict__ k, int k_stride, T* __restrict__ v, int v_stride, int rows, Divider per_row,
                  Divider lanes) {
  __shared__ Place place[MAX_ROWS];
  pdl_trigger();
  pdl_wait();
  const int r0 = blockIdx.x * rows, nr = min(rows, n_rows - r0), items = nr * (int)per_row.d;
  T *k0 = k + (long long)r0 * k_stride, *v0 = v + (long long)r0 * v_stride;
  find_places(place, P, r0, nr, cu, start, n_seq, page_table, max_pages);
  __syncthreads();
  for (int t0 = blockIdx.y * U * KV_THREADS + threadIdx.x; t0 < items; t0 += gridDim.y * U * KV_THREADS) {
    Raw<CT, PIECE<T>> raw[U];
    int byte[U];
    bool is_k[U];
    uint32_t r[U], h[U];
    Spots s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * KV_THREADS;
      if (t >= items) break;
      uint32_t col, i;
      per_row(t, r[u], col);
      lanes(col, h[u], i);
      s[u] = spots_of<PIECE<T>>(i, lanes.d, 0);
      const Place w = place[r[u]];
      is_k[u] = k && (int)h[u] < P.n_kv;
      if (k && !is_k[u]) h[u] -= P.n_kv;
      if (w.state != IN_POOL) continue;
      raw[u].load(static_cast<const CT*>(is_k[u] ? P.k : P.v) + w.at + (long long)h[u] * P.head_stride, s[u]);
      if constexpr (std::is_same<CT, e4m3_t>::value)
        byte[u] = (is_k[u] ? P.k_scale : P.v_scale)[w.scale_at + (h[u] << P.ps_shift)];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t0 + u * KV_THREADS >= items) break;
      const int state = place[r[u]].state;
      if (state == NO_SEQUENCE) continue;
      float a[8], b[8];
      if (state == IN_POOL) {
        values(raw[u], a, b);
        if constexpr (std::is_same<CT, e4m3_t>::value) {
          const float f = scale_of(byte[u]);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            a[e] *= f;
            b[e] *= f;
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] = b[e] = 0.f;
      }
      T* o = (is_k[u] ? k0 : v0) + (long long)r[u] * (is_k[u] ? k_stride : v_stride) + h[u] * P.head_dim;
      store8(o, s[u].x0, s[u].x1, a);
      store8(o, s[u].y0, s[u].y1, b);
    }
  }
}

template <typename F>
void by_type(rift_dtype dt, F f) {
  if (dt == RIFT_F32) f(float());
  else if (dt == RIFT_F16) f(__half());
  else f(__nv_bfloat16());
}
template <typename F>
void by_cache(rift_dtype dt, F f) {
  if (dt == RIFT_E4M3) f(e4m3_t());
  else if (dt == RIFT_F16) f(__half());
  else f(__nv_bfloat16());
}

}  // namespace

RopeAngles rope_angles(const rift_rope_spec& s, bool inverse) {
  RopeAngles R = {};
  R.rot_dim = s.rot_dim;
  R.interleaved = s.interleaved != 0;
  R.inverse = inverse;
  R.amplitude = (float)s.amplitude;
  R.amplitude_rest = (float)(s.amplitude - R.amplitude);
  R.ok = 1;
  double w[RIFT_ROPE_MAX_HEAD_DIM / 2];
  rope_frequencies(s, w);
  for (int j = 0; j < s.rot_dim / 2; ++j) {
    if (!(w[j] <= 2147483648.0)) R.ok = 0;
    else R.turns[j] = turns_of(w[j]);
  }
  return R;
}

// The launches are programmatic dependents of the kernel before them (each waits for it before its first access):
// they return whether the launch could be set up.
bool launch_rope(const void* x, rift_dtype dt, int n_rows, int n_heads, int head_dim, long long x_stride,
                 const int* positions, const RopeAngles& R, void* out, long long out_stride, cudaStream_t st) {
  bool ok = false;
  by_type(dt, [&](auto t) {
    ok = launch_rope_t<decltype(t)>(x, n_rows, n_heads, head_dim, x_stride, positions, R, out, out_stride, st);
  });
  return ok;
}

bool launch_kv_append(const KvPool& P, rift_dtype cache, const void* k, long long k_stride, const void* v,
                      long long v_stride, rift_dtype dt, int n_rows, const int* cu, const int* start, int n_seq,
                      const int* page_table, int max_pages, const RopeAngles* R, const void* q, long long q_stride,
                      int n_q, void* q_out, long long q_out_stride, cudaStream_t st) {
  const int lanes = P.head_dim / 16, per_row = (n_q + 2 * P.n_kv) * lanes;
  const int rows = rows_of_cta(n_rows, per_row, R ? R->rot_dim / 2 : 0, dt == RIFT_F32 ? 4 : 2);
  const dim3 grid(row_ctas(n_rows, rows), ctas_of_row(n_rows, per_row, U * KV_THREADS));
  const RopeAngles none = {};
  bool ok = false;
  by_type(dt, [&](auto t) {
    by_cache(cache, [&](auto c) {
      using T = decltype(t);
      ok = launch_ex(append_kernel<T, decltype(c)>, grid, dim3(KV_THREADS), 0, st, true, P, static_cast<const T*>(k),
                     (int)k_stride, static_cast<const T*>(v), (int)v_stride, n_rows, cu, start, n_seq, page_table, max_pages,
                     R != nullptr, R ? *R : none, static_cast<const T*>(q), (int)q_stride, n_q, static_cast<T*>(q_out),
                     (int)q_out_stride, rows, divider(per_row), divider(lanes), divider(R ? R->rot_dim / 2 : 1)) == cudaSuccess;
    });
  });
  return ok;
}

bool launch_kv_gather(const KvPool& P, rift_dtype cache, int n_rows, const int* cu, const int* start, int n_seq,
                      const int* page_table, int max_pages, void* k, long long k_stride, void* v, long long v_stride,
                      rift_dtype dt, cudaStream_t st) {
  const int lanes = P.head_dim / 16, per_row = ((k ? P.n_kv : 0) + (v ? P.n_kv : 0)) * lanes;
  const int rows = rows_of_cta(n_rows, per_row, 0, dt == RIFT_F32 ? 4 : 2);
  const dim3 grid(row_ctas(n_rows, rows), ctas_of_row(n_rows, per_row, U * KV_THREADS));
  bool ok = false;
  by_type(dt, [&](auto t) {
    by_cache(cache, [&](auto c) {
      using T = decltype(t);
      ok = launch_ex(gather_kernel<T, decltype(c)>, grid, dim3(KV_THREADS), 0, st, true, P, n_rows, cu, start, n_seq,
                     page_table, max_pages, static_cast<T*>(k), (int)k_stride, static_cast<T*>(v), (int)v_stride, rows,
                     divider(per_row), divider(lanes)) == cudaSuccess;
    });
  });
  return ok;
}

}  // namespace rift
