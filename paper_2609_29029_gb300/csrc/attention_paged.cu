// Attention of one new token per sequence over the paged KV cache (sm_103a).
//
// out = softmax(scale q K^T) V reads every cached row once and does 4 operations on each element and query
// head: HBM bounds it for any number of query heads that share a key head (a group) up to some tens.  So the
// kernel is built around the cache's stream: one CTA an SM, whose warps each copy tiles of keys and values
// into rings of their own (cp.async: a lane addresses its key's row through the page table, so a page may
// end anywhere in a tile), and compute on them while the next tiles arrive.
//
// The work is the list of all (sequence, key head, up to 8 NB query heads) items, cut into tiles of KT keys.  Every CTA
// takes the same number of consecutive tiles, but that a border inside a short item moves to the item's start (WHOLE_KEYS),
// and every warp the same share of its CTA's: sequences of any mix of lengths load the SMs about evenly, and no warp
// waits for another before its tiles are done.  A warp writes the items that it
// holds whole; the warps of a CTA join their parts of items, (reference, sum, output), at its end, and where an item is
// cut between CTAs, the one that brings the last part to the workspace joins them all (in the parts' order,
// whichever that is).
//
// Measured (device time): 16 sequences of 8,192 to 32,768 rows, 32 query heads over 8 of 128 in bf16, 179 us for 1.17 GB,
// 97% of the measured copy rate; 131,072 rows in e4m3 58 us for 271 MB (69%; 524,288 rows 84%, in pages of heads of rows
// 92%).  What does not grow with the rows is 12 us of the first and 13 to 16 of the second (lines through calls of four
// sizes): 4 to 5 before the first tile (lengths, pages and tiles, a DRAM latency each), as many behind the last, the rest
// not accounted for; what grows runs at 7.0 TB/s, and 6.1 or (heads of rows) 7.2: reads alone pass the rate of a copy.
// 73 sequences of 131 to 635 rows, 32 heads in fp16, 66 us for 384 MB; one of 635 rows 9 us.  A ring of two tiles ahead
// (128 KB an SM in flight) is what the rate takes; 16 KB tiles in four warps held the shorter sequences up (124 us for
// the 73).
//
// Per tile, with the keys as the rows of the products (16 keys x 8 query heads a tensor instruction, so that a
// group of up to 8 wastes nothing): S^T = K Q^T, the running maximum and sum per head, O^T += V^T P^T.  The
// products run on mma.sync: they take under a tenth of the time that a tile's bytes take to arrive, and the
// smallest tile of the tcgen05 unit (64 or 128 rows staged for one issuing thread) would add barriers between the
// warps of a stream that HBM bounds.
//  - K: the sum over a head's dims may go in any order, so a lane takes 16-byte chunks of its key's row as they lie,
//    and q's fragments are loaded in the same order.  Rows are stored with their chunks exclusive-ored by
//    the row, which keeps those loads and ldmatrix free of bank conflicts.
//  - V, 16 bits: ldmatrix.trans.  8 bits: a lane takes a chunk of 16 dims of four keys, pairs the bytes of
//    two keys, and converts them (exactly) to fp16.
//  - P: the 8 x 8 blocks of S^T transposed by movmatrix.
//  - e4m3 rows carry powers of two: K's multiplies the score (fp32, exact).  V's goes into the weight's exponent: the
//    weights in the product are 2^(s + e_v - M) with a running reference M of their own, so that each
//    keeps 11 bits whatever the other rows' scales are, beside l = sum 2^(s - m).
//  - weights of 16 bits would add their own rounding to the output's (in fp16 as much again, in bf16 ten times it):
//    they enter as the sum of two, at the price of a second product that the stream hides (no change in time).
//  - the products' sums are the tensor cores' own, which cut off below fp32's last bit at each step.  Before its rounding a long
//    bf16 output is off by some 10^-5: 0.33% of those of the 16 sequences are not the nearest value (0.06% of a plain fp32
//    form's).  Each 16 keys summed apart and a third bf16 number bring that to 0.03%, for 1 to 2% of the time there, 4
//    to 8% of short sequences' and up to 15% with 16 heads an item: not taken, beside a bf16 step of 0.4%.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kv_pages.cuh"
#include "paged_list.cuh"
#include "rift_internal.h"

namespace rift {

__device__ unsigned int g_err_paged;

unsigned int read_clear_err_paged() {
  unsigned int v = 0, z = 0;
  cudaMemcpyFromSymbol(&v, g_err_paged, sizeof(v));
  cudaMemcpyToSymbol(g_err_paged, &z, sizeof(z));
  return v;
}

namespace {

enum { CK_F16, CK_BF16, CK_E4M3 };

constexpr int WARPS = 8, THREADS = 32 * WARPS;
constexpr int MAX_CTAS = 160;    // one an SM
constexpr int STAGES = 3;        // tiles of a warp's ring
constexpr int SEQS = 1024;       // sequences whose lengths and tile counts a CTA holds at a time
// Items of up to this many keys, or up to an eighth of a CTA's share of tiles, are not cut between CTAs.  Joining an
// item's parts across CTAs takes 3 to 4 us behind the last tile, and an SM streams faster than its share of HBM while others
// have nothing left.  Both sides were measured at 540 points (1 to 24 sequences of 100 to 640 rows, 1, 8 and 32 key heads; fp16
// x 128, e4m3 x 64, bf16 x 128 in groups of 4): whole was never slower.  Cut and whole, us, fp16: one key head of 600 rows
// 11.5 and 8.6; 32 heads of 600 rows of 1, 5 and 10 sequences 10.7 and 9.7, 18.1 and 17.2 (the busiest CTA then has 76
// tiles for an even share of 40), 25.2 and 23.2.  Up to some 1,000 rows whole stays ahead at most points; at 2,500 rows of
// one head it takes 19.4 for 16.7.  Past SEQS sequences the borders' items would take a pass over the lengths to find, and a
// share holds several items in any case: borders stay where they fall.
constexpr int WHOLE_KEYS = 640;
// Weights are 2^(LIFT + s - m) for a running reference m that moves only when a score passes it by more than SLACK
// (a vote, instead of a reduction over the warp and a rescaling for every 16 keys): at most 2^15, which fp16 holds, and
// fp16 keeps all of its 11 bits down to 2^-23 of the reference (2^-14 for weights of at most one).  bf16 needs no lift, and its
// values may be so large (2^113 and more) that it takes the sums past fp32: DOWN, a power of two, brings those weights, and
// those that join parts, to one a key at most.
constexpr float LIFT = 9.f, SLACK = 6.f;
template <int CK>
constexpr float DOWN = CK == CK_BF16 ? 1.f / 32768.f : 1.f;

template <int HD, int CK, int NB>
struct Shape {
  static constexpr int ES = CK == CK_E4M3 ? 1 : 2;
  static constexpr int ROW = HD * ES, CPR = ROW / 16;  // bytes and 16-byte chunks of a key's row
  static constexpr int KT = 4096 / ROW;                // keys of a tile: 16, 32 or 64
  static constexpr int HALF = KT * ROW, STAGE = 2 * HALF;
  static constexpr int HG = 8 * NB;                    // query heads of an item
  static constexpr int RING = WARPS * STAGES * STAGE;
  static constexpr int SCALES = CK == CK_E4M3 ? WARPS * STAGES * 2 * KT * 4 : 0;
  static constexpr int SMEM = RING + SCALES;
};

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool real) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_end_group() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];\n" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void ldmatrix_trans(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(r) : "r"(v));
  return r;
}
template <bool BF16>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (BF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 2^x to 2^-22 (2^-inf = 0; a NaN stays one).
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) { return __byte_perm(a, b, sel); }

// Byte offset of chunk c of row r of a tile.
template <int CPR>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) {
  if (CPR >= 8) return (uint32_t)(r * CPR + (c ^ (r & 7))) * 16u;
  const int line = r >> 1;  // two rows of four chunks share 128 bytes
  return (uint32_t)(line * 8 + ((((r & 1) << 2) | c) ^ (line & 7))) * 16u;
}
// The j-th chunk of a key's row that lane (., t) takes.
template <int CPR>
__device__ __forceinline__ int chunk_of(int j, int t) {
  return CPR >= 8 ? 2 * t + (j & 1) + 8 * (j >> 1) : t;
}

struct Args {
  KvPool P;
  // the pool's strides in units of `unit` bytes, a power of two that divides them: a row's offset fits 32 bits
  uint32_t page_u, row_u, head_u, unit, scale_page;  // scale_page: scale bytes of a page
  const void* q;
  long long q_stride;
  int n_heads, group, hblocks;  // query heads; those of a key head; items of a key head
  const int* seq_lens;
  int n_seq;
  const int* page_table;
  int max_pages, window;
  float scale_log2;
  void* out;
  long long out_stride;
  float* lse;
  float* part_o;    // [MAX_CTAS][WARPS][HG][HD]: outputs of the parts of items that warps end early with
  float* cta_o;     // [MAX_CTAS][2][HG][HD]: outputs of CTAs' parts of items
  float2* cta_ml;   // [MAX_CTAS][2][HG]: their references (log2 units) and sums
  unsigned long long* arrived;  // [MAX_CTAS][2]: the parts of an item that are in place, counted at its first CTA
  int q_bf16;
};

// A sequence's length as it counts: 0 where it is out of range (reported by the caller that is told to).
__device__ __forceinline__ int length_of(const Args& A, int i, bool report) {
  const int L = A.seq_lens[i];
  if (L >= 0 && L <= ((long long)A.max_pages << A.P.ps_shift)) return L;
  if (report) atomicOr(&g_err_paged, RIFT_EBIT_CAPACITY);
  return 0;
}
__device__ __forceinline__ int first_key(int L, int window) { return window > 0 ? max(0, L - window) : 0; }
template <int KT>
__device__ __forceinline__ int tiles_of(int L, int window) {
  return (L + KT - 1) / KT - first_key(L, window) / KT;
}

// A position in the list of items: an item is (sequence, key head, block of query heads).
template <int KT>
struct Items {
  int seq, head, blk, L, lo, t0, n;  // keys lo .. L - 1; first tile and tiles of the item
  long long base;                    // tiles of the items before it
  __device__ __forceinline__ void load(const Args& A, const int* lens) {
    L = A.n_seq <= SEQS ? lens[seq] : length_of(A, seq, false);
    lo = first_key(L, A.window);
    t0 = lo / KT;
    n = (L + KT - 1) / KT - t0;
  }
  // On to the next item that has tiles; only called where there is one (seq == n_seq past the last).
  __device__ __forceinline__ void next(const Args& A, const int* lens) {
    base += n;
    if (++blk < A.hblocks) return;
    blk = 0;
    if (++head < A.P.n_kv) return;
    head = 0;
    do {
      if (++seq >= A.n_seq) {
        n = 0;
        return;
      }
      load(A, lens);
    } while (n == 0);
  }
};

__device__ __forceinline__ uint16_t bits16(float v, int bf16) {
  return bf16 ? __bfloat16_as_ushort(__float2bfloat16_rn(v)) : __half_as_ushort(__float2half_rn(v));
}
constexpr float LN2 = 0.6931471805599453f;
// What a weight's exponent counts from; no score above -inf yet: 0, whose weights are 2^-inf.
__device__ __forceinline__ float reference(float m) { return m == -INFINITY ? 0.f : m - LIFT; }

// Counts one more of `parts` arrivals at an item, in two words of the workspace: whether it was the last.  word[0] holds
// KEY above the count, and the last arrival leaves a count of zero behind it, so that every call but a workspace's
// first finds zero.  What a workspace holds before that lacks the key (one word in 2^48 would not), and goes on
// lacking it while the arrivals of that call are added to it: they all count again in word[1], by exchanges, which
// are slow where many meet (20 parts: 7 us), but tell a word without the key from a count.
constexpr unsigned long long KEY = 0x5bd1e995a3c7ull << 16;
__device__ __forceinline__ bool has_key(unsigned long long w) { return (w & ~0xffffull) == KEY; }
__device__ __forceinline__ bool arrive(unsigned long long* word, int parts) {
  const unsigned long long was = atomicAdd(word, 1ull);
  if (has_key(was)) {
    if ((int)(was & 0xffffull) + 1 != parts) return false;
    atomicExch(word, KEY);
    return true;
  }
  unsigned long long seen = KEY;
  for (;;) {
    const unsigned n = has_key(seen) ? (unsigned)(seen & 0xffffull) + 1 : 1u;
    const unsigned long long put = KEY | (n == (unsigned)parts ? 0u : n), then = atomicCAS(word + 1, seen, put);
    if (then == seen) {
      if (n != (unsigned)parts) return false;
      atomicExch(word, KEY);
      return true;
    }
    seen = then;
  }
}

// A warp's part of an item that it does not hold whole.
struct Part {
  int seq, head, blk, n;  // the item (seq -1: none) and its tiles
  long long base;
  int early;              // where its output is, [HG][HD] over the sum: 1 the workspace, 0 the warp's ring
};
constexpr int PARTS = 2 * WARPS;  // at most two a warp: one of an item that began before its tiles, one of an item that
                                  // goes on behind them

template <int HD, int CK, int NB>
__global__ void __launch_bounds__(THREADS, 1) paged_attn_kernel(const __grid_constant__ Args A) {
  using S = Shape<HD, CK, NB>;
  constexpr int KT = S::KT, CPR = S::CPR, MB = KT / 16, KW = KT > 32 ? KT / 32 : 1, DT = HD / 16, QW = HD / 8;
  constexpr uint32_t WHOLE = KT >= 32 ? 0xffffffffu : (1u << KT) - 1;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ long long scan[33], before[SEQS + 1];
  __shared__ int lens[SEQS];
  __shared__ uint32_t masks[WARPS][STAGES][KW];
  __shared__ Part parts[PARTS];
  __shared__ float2 part_ml[PARTS][S::HG];  // references (log2 units) and sums
  __shared__ float part_w[PARTS][S::HG], run_m[PARTS][S::HG];
  __shared__ int run[PARTS];
  __shared__ Part cut[2];  // what goes on in other CTAs: the item that began before, the one that goes on behind
  __shared__ int last[2], span[2][2];  // whether this CTA brought the item's last part; its first and last CTA
  static_assert(S::SMEM + sizeof(scan) + sizeof(before) + sizeof(lens) + sizeof(masks) + sizeof(parts) + sizeof(part_ml) +
                        sizeof(part_w) + sizeof(run_m) + sizeof(run) + sizeof(cut) + sizeof(last) + sizeof(span) + 256 <=
                    227 * 1024,
                "the shared memory of an SM (256: the arrays' alignment)");
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int per_seq = A.P.n_kv * A.hblocks;
  const int q_bf16 = CK == CK_BF16 ? 1 : CK == CK_F16 ? 0 : A.q_bf16;
  pdl_trigger();
  pdl_wait();
  // ---- the list's tiles: lengths, and tiles before each sequence (of SEQS at a time; a copy a warp of up to 32, which
  // needs no barrier)
  const bool few = A.n_seq <= 32;
  int* len = lens + (few ? 32 * warp : 0);
  long long* tiles_before = before + (few ? 32 * warp : 0);
  auto fill = [&](int s0) {
    long long sum = 0;
    const int m = min(SEQS, A.n_seq - s0);
    for (int i0 = 0; i0 < m; i0 += THREADS) {
      const int i = i0 + tid;
      const int L = i < m ? length_of(A, s0 + i, blockIdx.x == 0) : 0;
      long long total;
      const long long at = sum + block_excl_scan<long long>(tiles_of<KT>(L, A.window), scan, &total);
      if (i < m) {
        lens[i] = L;
        before[i] = at;
      }
      sum += total;
    }
    __syncthreads();
    return sum;
  };
  long long W = 0;
  if (few) {
    const int L = lane < A.n_seq ? length_of(A, lane, blockIdx.x == 0 && warp == 0) : 0;
    const long long n = tiles_of<KT>(L, A.window), to = warp_incl_scan(n);
    len[lane] = L;
    tiles_before[lane] = to - n;
    W = __shfl_sync(0xffffffffu, to, 31);
    __syncwarp();
  } else {
    for (int s0 = 0; s0 < A.n_seq; s0 += SEQS) W += fill(s0);
  }
  W *= per_seq;
  const int c = blockIdx.x, G = gridDim.x;
  auto tiles = [&](int i) { return tiles_of<KT>(len[i], A.window); };

  // ---- the CTA's tiles [c0, c1) of the list, and the warp's [u0, u1) of them
  const Shares ctas(W, G);
  long long c0 = ctas.begin(c), c1 = ctas.begin(c + 1), u0, u1;
  auto cut_for_warps = [&]() {
    const long long T = c1 - c0, each = T >= WARPS ? T / WARPS : 1, more = T >= WARPS ? T % WARPS : 0;
    u0 = min(c1, c0 + each * warp + min((long long)warp, more));
    u1 = min(c1, u0 + each + (warp < more ? 1 : 0));
  };
  Items<KT> it;
  it.seq = -1;
  if (A.n_seq <= SEQS) {
    u0 = u1 = 0;
    if (W > 0) {
#pragma unroll 1
      for (int pass = 0; pass < 2; ++pass) {  // the item that holds tile x: the CTA's borders (a lane each), then u0
        const long long x = pass == 0 ? (lane & 1 ? c1 : c0) : u0;
        const ListItem at = item_at(x, W, per_seq, tiles_before, A.n_seq, tiles);
        if (pass == 0) {
          const long long to = x >= W || at.n > max((long long)(WHOLE_KEYS / KT), ctas.each / 8) ? x : at.base;
          c0 = __shfl_sync(0xffffffffu, to, 0);
          c1 = __shfl_sync(0xffffffffu, to, 1);
          cut_for_warps();
        } else {
          it.seq = at.seq;
          it.base = at.base;
          it.head = A.hblocks == 1 ? at.block : at.block / A.hblocks;
          it.blk = at.block - it.head * A.hblocks;
        }
      }
    }
  } else {
    cut_for_warps();
    long long passed = 0;
    for (int s0 = 0; s0 < A.n_seq; s0 += SEQS) {
      __syncthreads();
      const int m = min(SEQS, A.n_seq - s0);
      const long long sum = fill(s0), x = u0 - passed * per_seq;
      if (u0 < u1 && it.seq < 0 && x < sum * per_seq) {
        const ListItem at = item_at(x, sum * per_seq, per_seq, tiles_before, m, tiles);
        it.seq = s0 + at.seq;
        it.base = passed * per_seq + at.base;
        it.head = at.block / A.hblocks;
        it.blk = at.block % A.hblocks;
      }
      passed += sum;
    }
  }
  const bool any = u0 < u1;
  if (any) it.load(A, len);

  // ---- the warp's ring: tile u of the worker's range in slot (u - u0) % STAGES
  const uint32_t ring = smem_addr(smem) + warp * STAGES * S::STAGE;
  float* scale_ring = reinterpret_cast<float*>(smem + S::RING) + warp * STAGES * 2 * KT;  // K's factors, V's exponents
  // the chunk of a row that this lane copies: its place in the pools' rows, and in a tile's first rows
  const uint8_t* klane = static_cast<const uint8_t*>(A.P.k) + lane % CPR * 16;
  const uint8_t* vlane = static_cast<const uint8_t*>(A.P.v) + lane % CPR * 16;
  const uint32_t to_lane = chunk_at<CPR>(lane / CPR, lane % CPR);
  struct Tile {  // a tile to copy: its keys' pages (a key a lane, -1: none), first key, the item's keys and key head
    int pg[KW];
    int key0, lo, L, head;
  };
  Items<KT> ld = it;  // the item of the next tile to look up, which tile of it, how many there are to come
  int lt = any ? (int)(u0 - it.base) : 0;
  long long to_come = u1 - u0;
  auto look_up = [&]() {
    Tile x;
    x.L = 0;
    if (to_come <= 0) return x;
    --to_come;
    if (lt >= ld.n) {
      ld.next(A, len);
      lt = 0;
    }
    x.key0 = (ld.t0 + lt) * KT;
    ++lt;
    x.lo = ld.lo;
    x.L = ld.L;
    x.head = ld.head;
    const int* pages = A.page_table + (long long)ld.seq * A.max_pages;
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      const int key = x.key0 + 32 * w + lane;
      x.pg[w] = lane < KT && key >= x.lo && key < x.L ? pages[key >> A.P.ps_shift] : -1;
    }
    return x;
  };
  // e4m3: the scale bytes of the last copied tile, on their way: they go to shared memory with the next tile's copies,
  // so that no warp waits for them
  uint32_t sc_k[KW], sc_v[KW];
  int sc_slot = -1, put = 0;
  auto issue = [&](const Tile& x) {  // the tile's copies into slot `put`, as one group (empty past the end)
    if constexpr (CK == CK_E4M3) {
      if (sc_slot >= 0) {
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          scale_ring[sc_slot * 2 * KT + 32 * w + lane] = scale_of(sc_k[w]);
          scale_ring[sc_slot * 2 * KT + KT + 32 * w + lane] = (float)((int)sc_v[w] - 127);
        }
        sc_slot = -1;
      }
    }
    if (x.L > 0) {
      uint32_t off[KW], real[KW], all = WHOLE;
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const int key = x.key0 + 32 * w + lane, row = key & ((1 << A.P.ps_shift) - 1);
        const bool in = lane < KT && key >= x.lo && key < x.L, ok = in && (uint32_t)x.pg[w] < (uint32_t)A.P.n_pages;
        if (in && !ok) atomicOr(&g_err_paged, RIFT_EBIT_BADID);
        off[w] = ok ? x.pg[w] * A.page_u + row * A.row_u + x.head * A.head_u : 0u;
        if constexpr (CK == CK_E4M3) {
          const unsigned long long at = ok ? (unsigned long long)(uint32_t)x.pg[w] * A.scale_page + ((x.head << A.P.ps_shift) + row) : 0;
          sc_k[w] = A.P.k_scale[at];
          sc_v[w] = A.P.v_scale[at];
        }
        real[w] = __ballot_sync(0xffffffffu, ok);
        all &= real[w];
        if (lane == 0) masks[warp][put][w] = real[w];
      }
      sc_slot = put;
      // copy k of the warp: rows k RPC + lane / CPR, a chunk a lane.  Row r's chunk c lies at c ^ (r & 7); with q = lane / CPR
      // that is (c ^ q) ^ (k RPC & 7), as RPC rows are a power of two of them.
      constexpr int RPC = 32 / CPR;
      const uint32_t dst = ring + put * S::STAGE;
      auto copies = [&](auto whole) {
#pragma unroll
        for (int k = 0; k < KT / RPC; ++k) {
          const uint32_t o = __shfl_sync(0xffffffffu, off[k * RPC / 32], (k * RPC & 31) + lane / CPR);
          const unsigned long long from = (unsigned long long)o * A.unit;
          const uint32_t d = CPR >= 8 ? dst + k * RPC * S::ROW + (to_lane ^ ((k * RPC & 7) * 16))
                                      : dst + chunk_at<CPR>(k * RPC + lane / CPR, lane % CPR);
          if constexpr (decltype(whole)::value) {
            copy16(d, klane + from);
            copy16(d + S::HALF, vlane + from);
          } else {
            const bool ok = real[k * RPC / 32] >> ((k * RPC & 31) + lane / CPR) & 1u;
            copy16(d, klane + from, ok);
            copy16(d + S::HALF, vlane + from, ok);
          }
        }
      };
      if (all == WHOLE) copies(std::true_type());
      else copies(std::false_type());
    }
    copies_end_group();
    put = put + 1 == STAGES ? 0 : put + 1;
  };

  // ---- queries: the fragments of the next item, fetched while the present one is worked on
  uint32_t qn[NB][QW], qf[NB][QW];
  auto fetch_q = [&](const Items<KT>& x) {
    const int h0 = x.blk * S::HG;
    const uint16_t* row = static_cast<const uint16_t*>(A.q) + x.seq * A.q_stride + (long long)x.head * A.group * HD;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int h = h0 + 8 * b + g;
      const bool real = h < A.group;
#pragma unroll
      for (int w = 0; w < QW / 4; ++w) {  // 16 bytes: 8 dims
        const int dim = CK == CK_E4M3 ? 16 * chunk_of<CPR>(w / 2, t) + 8 * (w & 1) : 8 * chunk_of<CPR>(w, t);
        const uint4 v = real ? *reinterpret_cast<const uint4*>(row + (long long)h * HD + dim) : make_uint4(0u, 0u, 0u, 0u);
        qn[b][4 * w] = v.x;
        qn[b][4 * w + 1] = v.y;
        qn[b][4 * w + 2] = v.z;
        qn[b][4 * w + 3] = v.w;
      }
    }
  };

  Tile ahead;  // looked up, to be copied next
  if (any) {
    ahead = look_up();
    fetch_q(it);
#pragma unroll 1
    for (int s = 0; s < STAGES - 1; ++s) {
      issue(ahead);
      ahead = look_up();
    }
  }
  // sequences without rows: zeros, while the first tiles arrive
  for (int i = blockIdx.x; i < A.n_seq; i += gridDim.x) {
    if ((A.n_seq <= SEQS ? len[i] : length_of(A, i, false)) > 0) continue;
    uint16_t* o = static_cast<uint16_t*>(A.out) + i * A.out_stride;
    for (int k = tid; k < A.n_heads * HD; k += THREADS) o[k] = 0;
    if (A.lse)
      for (int k = tid; k < A.n_heads; k += THREADS) A.lse[(long long)i * A.n_heads + k] = -INFINITY;
  }
  if (lane < 2) parts[2 * warp + lane].seq = -1;
  __syncwarp();

  long long u = u0;
  int slot = 0;
  while (u < u1) {
    const long long part_lo = u, part_hi = min(it.base + it.n, u1);
    // heads 2t and 2t + 1 of each block of 8: score factor, running maxima, this lane's share of the sum
    float f[NB][2], m[NB][2], mv[NB][2], l[NB][2], o[DT][NB][4], from[NB][2], from_v[NB][2];  // from: reference(m)
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      f[b][0] = f[b][1] = A.scale_log2;
      if (CK == CK_E4M3 && q_bf16) {  // bf16 queries as fp16 times a power of two that brings the head's largest to 2^14 .. 2^15
        float top = 0.f;
#pragma unroll
        for (int w = 0; w < QW; ++w) {
          const float lo = fabsf(__uint_as_float(qn[b][w] << 16)), hi = fabsf(__uint_as_float(qn[b][w] & 0xffff0000u));
          top = fmaxf(top, fmaxf(lo <= 3.402823466e38f ? lo : 0.f, hi <= 3.402823466e38f ? hi : 0.f));
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int e = min(max((int)(__float_as_uint(top) >> 23), 15), 254);  // top ~ 2^(e - 127)
        const float down = __uint_as_float((uint32_t)(268 - e) << 23), up = __uint_as_float((uint32_t)max(e - 14, 1) << 23);
#pragma unroll
        for (int w = 0; w < QW; ++w)
          qf[b][w] = pack_half2(__uint_as_float(qn[b][w] << 16) * down, __uint_as_float(qn[b][w] & 0xffff0000u) * down);
        f[b][0] *= __shfl_sync(0xffffffffu, up, 8 * t);
        f[b][1] *= __shfl_sync(0xffffffffu, up, 8 * t + 4);
      } else {
#pragma unroll
        for (int w = 0; w < QW; ++w) qf[b][w] = qn[b][w];
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        m[b][e] = mv[b][e] = -INFINITY;
        from[b][e] = from_v[b][e] = 0.f;
        l[b][e] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][b][e] = 0.f;
    }
    Items<KT> nx = it;
    if (part_hi < u1) {
      nx.next(A, len);
      fetch_q(nx);
    }

    for (; u < part_hi; ++u) {
      copies_wait<STAGES - 2>();
      __syncwarp();  // the tile is whole, and every lane is done with the slot that is filled next
      issue(ahead);
      ahead = look_up();
      const uint32_t kt = ring + slot * S::STAGE, vt = kt + S::HALF;
      const uint32_t* mask = masks[warp][slot];
      const float* scales = scale_ring + slot * 2 * KT;
      slot = slot + 1 == STAGES ? 0 : slot + 1;

#pragma unroll 1
      for (int a = 0; a < MB; ++a) {  // 16 keys: this lane's scores are those of keys g and g + 8
        const uint32_t real = mask[a >> 1] >> (16 * (a & 1)) & 0xffffu;
        if (real == 0u) continue;
        const uint32_t ka = kt + chunk_at<CPR>(16 * a, 0), va = vt + chunk_at<CPR>(16 * a, 0);
        // S^T = K Q^T; two sums a head block, so that the products wait for each other half as often
        float s[NB][4], s2[NB][4];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[b][e] = s2[b][e] = 0.f;
#pragma unroll
        for (int j = 0; j < CPR / 4; ++j) {
          const int ch = chunk_of<CPR>(j, t);
          const uint4 x = lds16(ka + chunk_at<CPR>(g, ch)), y = lds16(ka + chunk_at<CPR>(8 + g, ch));
          const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
          if (CK == CK_E4M3) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              uint32_t a0, a1, a2, a3;
              half2s_of(xw[k], a0, a2);
              half2s_of(yw[k], a1, a3);
#pragma unroll
              for (int b = 0; b < NB; ++b)
                mma<false>(k & 1 ? s2[b] : s[b], a0, a1, a2, a3, qf[b][8 * j + 2 * k], qf[b][8 * j + 2 * k + 1]);
            }
          } else {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int b = 0; b < NB; ++b)
                mma<CK == CK_BF16>(k & 1 ? s2[b] : s[b], xw[2 * k], yw[2 * k], xw[2 * k + 1], yw[2 * k + 1], qf[b][4 * j + 2 * k],
                                   qf[b][4 * j + 2 * k + 1]);
          }
        }
        // scores in log2 units; whether one passes its reference
        float ev[2];
        bool passes = false;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const bool in = real >> (8 * r + g) & 1u;
          float ks = 1.f;
          if (CK == CK_E4M3) {
            ks = scales[16 * a + 8 * r + g];
            ev[r] = scales[KT + 16 * a + 8 * r + g];
          }
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float& v = s[b][2 * r + e];
              v += s2[b][2 * r + e];
              v = in ? (CK == CK_E4M3 ? v * (ks * f[b][e]) : v * f[b][e]) : -INFINITY;
              passes |= v > m[b][e] + SLACK;
              if (CK == CK_E4M3) passes |= v + ev[r] > mv[b][e] + SLACK;
            }
        }
        if (__any_sync(0xffffffffu, passes)) {
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float top = fmaxf(m[b][e], fmaxf(s[b][e], s[b][2 + e])), topv = 0.f;
              if (CK == CK_E4M3) topv = fmaxf(mv[b][e], fmaxf(s[b][e] + ev[0], s[b][2 + e] + ev[1]));
#pragma unroll
              for (int d = 4; d < 32; d <<= 1) {
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                if (CK == CK_E4M3) topv = fmaxf(topv, __shfl_xor_sync(0xffffffffu, topv, d));
              }
              // (a head without a score above -inf yet has nothing to rescale)
              const float down = top == -INFINITY ? 1.f : ex2(m[b][e] - top);
              l[b][e] *= down;
              m[b][e] = top;
              from[b][e] = reference(top);
              float down_o = down;
              if (CK == CK_E4M3) {
                down_o = topv == -INFINITY ? 1.f : ex2(mv[b][e] - topv);
                mv[b][e] = topv;
                from_v[b][e] = reference(topv);
              }
#pragma unroll
              for (int i = 0; i < DT; ++i) {
                o[i][b][e] *= down_o;
                o[i][b][2 + e] *= down_o;
              }
            }
        }
        // weights
        uint32_t p[NB][2], p2[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float w[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float v = s[b][2 * r + e];
              const float x = ex2(v - from[b][e]);
              l[b][e] += x;
              w[e] = CK == CK_E4M3 ? ex2(v + ev[r] - from_v[b][e]) : x * DOWN<CK>;
            }
            if (CK == CK_BF16) {
              const uint32_t hi = pack_bf16x2(w[0], w[1]);
              p[b][r] = transpose8(hi);
              p2[b][r] = transpose8(pack_bf16x2(w[0] - __uint_as_float(hi << 16), w[1] - __uint_as_float(hi & 0xffff0000u)));
            } else {
              const uint32_t hi = pack_half2(w[0], w[1]);
              const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&hi));
              p[b][r] = transpose8(hi);
              p2[b][r] = transpose8(pack_half2(w[0] - back.x, w[1] - back.y));
            }
          }
        // O^T += V^T P^T
        if (CK == CK_E4M3) {
          constexpr int VW = HD / 32;  // words of a lane's dims of a key
          uint32_t v[4][VW];           // keys 2t, 2t + 1, 2t + 8, 2t + 9
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int row = 2 * t + (k & 1) + 8 * (k >> 1);
            if constexpr (HD == 128) {
              const uint4 x = lds16(va + chunk_at<CPR>(row, g));
              v[k][0] = x.x;
              v[k][1] = x.y;
              v[k][2] = x.z;
              v[k][3] = x.w;
            } else {
              const uint2 x = lds8(va + chunk_at<CPR>(row, g >> 1) + 8 * (g & 1));
              v[k][0] = x.x;
              v[k][1] = x.y;
            }
          }
#pragma unroll
          for (int i = 0; i < DT; ++i) {  // dims (HD / 8) g + 2 i and + 1
            const uint32_t sel = i & 1 ? 0x7362 : 0x5140;  // bytes 2i, 2i + 1 of both keys of a pair
            const uint32_t x = prmt(v[0][i / 2], v[1][i / 2], sel), y = prmt(v[2][i / 2], v[3][i / 2], sel);
            uint32_t a0, a1, a2, a3;
            half2s_of(x, a0, a1);
            half2s_of(y, a2, a3);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
              mma<false>(o[i][b], a0, a1, a2, a3, p[b][0], p[b][1]);
              mma<false>(o[i][b], a0, a1, a2, a3, p2[b][0], p2[b][1]);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < DT; ++i) {  // dims 16 i + g and + 8
            uint32_t v[4];
            ldmatrix_trans(v, va + chunk_at<CPR>((lane & 7) + ((lane >> 4) & 1) * 8, 2 * i + ((lane >> 3) & 1)));
#pragma unroll
            for (int b = 0; b < NB; ++b) {
              mma<CK == CK_BF16>(o[i][b], v[0], v[1], v[2], v[3], p[b][0], p[b][1]);
              mma<CK == CK_BF16>(o[i][b], v[0], v[1], v[2], v[3], p2[b][0], p2[b][1]);
            }
          }
        }
      }
    }

    // ---- the item's output, or this part of it
    const int kvh = it.head, h0 = it.blk * S::HG, hn = min(S::HG, A.group - h0);
    const bool starts = part_lo == it.base, ends = part_hi == it.base + it.n, whole = starts && ends;
    const int mine = 2 * warp + (starts ? 1 : 0);
    // the warp's last part goes where its ring was, an earlier one to the workspace
    float* part = part_hi == u1 ? reinterpret_cast<float*>(smem + warp * STAGES * S::STAGE)
                                : A.part_o + ((long long)c * WARPS + warp) * S::HG * HD;
    if (part_hi == u1) {
      copies_wait<0>();
      __syncwarp();
    }
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[b][e] += __shfl_xor_sync(0xffffffffu, l[b][e], d);
        const int h = 8 * b + 2 * t + e;
        if (h >= hn) continue;
        const float sum = l[b][e], M = reference(m[b][e]);
        // no key at all (bad pages, scores of -inf): zero; e4m3 outputs stand relative to their own reference
        const float to_y = sum == 0.f ? 0.f : (CK == CK_E4M3 ? exp2f(reference(mv[b][e]) - M) : 1.f / DOWN<CK>) / sum;
        const long long head = (long long)kvh * A.group + h0 + h;
        if (whole) {
          uint16_t* dst = static_cast<uint16_t*>(A.out) + it.seq * A.out_stride + head * HD;
#pragma unroll
          for (int i = 0; i < DT; ++i) {
            const int d0 = CK == CK_E4M3 ? HD / 8 * g + 2 * i : 16 * i + g, d1 = CK == CK_E4M3 ? d0 + 1 : d0 + 8;
            dst[d0] = bits16(o[i][b][e] * to_y, q_bf16);
            dst[d1] = bits16(o[i][b][2 + e] * to_y, q_bf16);
          }
          if (A.lse && g == 0)
            A.lse[(long long)it.seq * A.n_heads + head] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * LN2;
        } else {
          float* dst = part + h * HD;
#pragma unroll
          for (int i = 0; i < DT; ++i) {
            const int d0 = CK == CK_E4M3 ? HD / 8 * g + 2 * i : 16 * i + g, d1 = CK == CK_E4M3 ? d0 + 1 : d0 + 8;
            dst[d0] = o[i][b][e] * to_y;
            dst[d1] = o[i][b][2 + e] * to_y;
          }
          if (g == 0) part_ml[mine][h] = make_float2(M, sum);
        }
      }
    if (!whole && lane == 0) parts[mine] = Part{it.seq, it.head, it.blk, it.n, it.base, part_hi < u1};
    it = nx;
  }
  copies_wait<0>();

  // ---- the CTA's warps' parts joined: a run of parts of one item, in the warps' order
  // (Every step behind the last tile waits for the one before it, so each puts all of its loads out at once.)
  if (tid < 2) cut[tid].seq = -1;
  __syncthreads();
  uint32_t valid, leads, early;  // the parts there are; those that begin a run; those in the workspace
  {
    const bool is = lane < PARTS && parts[lane & (PARTS - 1)].seq >= 0;
    const long long base = is ? parts[lane].base : -1;
    valid = __ballot_sync(0xffffffffu, is);
    early = __ballot_sync(0xffffffffu, is && parts[lane & (PARTS - 1)].early);
    const uint32_t before_it = valid & ((1u << lane) - 1);
    const long long prior = __shfl_sync(0xffffffffu, base, before_it ? 31 - __clz(before_it) : 0);
    const bool lead = is && (before_it == 0u || prior != base);
    leads = __ballot_sync(0xffffffffu, lead);
    if (warp == 0 && lead) run[__popc(leads & ((1u << lane) - 1))] = lane;
  }
  auto run_of = [&](int k) {  // the parts of the run that part k begins
    const uint32_t later = leads & ~((2u << k) - 1);
    return valid & ((later ? later & -later : 1u << PARTS) - (1u << k));
  };
  for (int x = tid; x < PARTS * S::HG; x += THREADS) {  // each part's weight in its item, a head a thread
    const int i = x / S::HG, h = x % S::HG;
    if (!(valid >> i & 1u) || h >= A.group - parts[i].blk * S::HG) continue;
    const int k = 31 - __clz(leads & ((2u << i) - 1));
    const uint32_t members = run_of(k);
    float M = -INFINITY;
#pragma unroll
    for (int j = 0; j < PARTS; ++j) {
      const float2 y = part_ml[j][h];
      if ((members >> j & 1u) && y.y != 0.f) M = fmaxf(M, y.x);
    }
    const float2 y = part_ml[i][h];
    part_w[i][h] = y.y == 0.f ? 0.f : y.y * exp2f(y.x - M) * DOWN<CK>;
    run_m[i][h] = M;
  }
  if (tid >= THREADS - 2 && leads) {  // only the first run can have begun before the CTA's tiles, only the last go on
    const int which = tid - (THREADS - 2);
    const Part& p = parts[which == 0 ? __ffs(leads) - 1 : 31 - __clz(leads)];
    const bool starts = p.base >= c0, ends = p.base + p.n <= c1;
    if (which == 0 ? !starts : starts && !ends) {
      cut[which] = p;
      span[which][0] = ctas.owner(p.base);
      span[which][1] = ctas.owner(p.base + p.n - 1);
    }
  }
  __syncthreads();
  const int quads = min(S::HG, A.group) * (HD / 4);  // of a run, four elements each
  for (int x = tid; x < __popc(leads) * quads; x += THREADS) {
    const int r = (int)((uint32_t)x / (uint32_t)quads), y4 = 4 * (x - r * quads), h = y4 / HD, d = y4 % HD;
    const int k = run[r];
    const uint32_t members = run_of(k);
    const Part& p = parts[k];
    const int h0 = p.blk * S::HG;
    const bool starts = p.base >= c0, ends = p.base + p.n <= c1, whole = starts && ends;
    if (h >= A.group - h0) continue;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < PARTS; ++j) {
      if (!(members >> j & 1u)) continue;
      const float* o = early >> j & 1u ? A.part_o + ((long long)c * WARPS + j / 2) * S::HG * HD
                                       : reinterpret_cast<const float*>(smem + j / 2 * STAGES * S::STAGE);
      const float4 y = *reinterpret_cast<const float4*>(o + y4);
      const float w = part_w[j][h];
      if (w == 0.f) continue;
      sum += w;
      acc.x = fmaf(w, y.x, acc.x);
      acc.y = fmaf(w, y.y, acc.y);
      acc.z = fmaf(w, y.z, acc.z);
      acc.w = fmaf(w, y.w, acc.w);
    }
    const float M = run_m[k][h], inv = sum == 0.f ? 0.f : 1.f / sum;
    const long long head = (long long)p.head * A.group + h0 + h;
    if (whole) {
      uint16_t* dst = static_cast<uint16_t*>(A.out) + p.seq * A.out_stride + head * HD + d;
      *reinterpret_cast<ushort4*>(dst) = make_ushort4(bits16(acc.x * inv, q_bf16), bits16(acc.y * inv, q_bf16),
                                                      bits16(acc.z * inv, q_bf16), bits16(acc.w * inv, q_bf16));
      if (A.lse && d == 0)
        A.lse[(long long)p.seq * A.n_heads + head] = sum == 0.f ? -INFINITY : (M + log2f(sum / DOWN<CK>)) * LN2;
    } else {
      const long long at = (2LL * c + (starts ? 1 : 0)) * S::HG + h;
      *reinterpret_cast<float4*>(A.cta_o + at * HD + d) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
      if (d == 0) A.cta_ml[at] = make_float2(M, sum / DOWN<CK>);
    }
  }

  // ---- items cut between CTAs: whoever brings the last part joins them
  if (cut[0].seq < 0 && cut[1].seq < 0) return;
  __syncthreads();
  if (tid < 2) {
    last[tid] = 0;
    if (cut[tid].seq >= 0) {
      __threadfence();  // the CTA's parts before the count
      last[tid] = arrive(A.arrived + 2 * span[tid][0], span[tid][1] - span[tid][0] + 1);
      __threadfence();  // the count before the others' parts
    }
  }
  __syncthreads();
  float* weight = reinterpret_cast<float*>(smem);  // [parts][HG], where the rings were
  static_assert(MAX_CTAS * S::HG * 4 <= S::RING, "");
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {
    if (!last[k]) continue;
    const Part p = cut[k];
    const int first = span[k][0], n = span[k][1] - first + 1;
    const int h0 = p.blk * S::HG, hn = min(S::HG, A.group - h0);
    auto at = [&](int i) { return (2LL * (first + i) + (i == 0 ? 1 : 0)) * S::HG; };
    auto part = [&](int i, int x) { return __ldcg(reinterpret_cast<const float4*>(A.cta_o + at(i) * HD + x)); };
    constexpr int FIRST = 16;  // parts whose outputs are on their way while the weights are worked out
    float4 y[FIRST];
#pragma unroll
    for (int i = 0; i < FIRST; ++i)
      if (i < n && 4 * tid < hn * HD) y[i] = part(i, 4 * tid);
    for (int h = warp; h < hn; h += WARPS) {  // the parts' weights, a head a warp
      float M = -INFINITY, sum = 0.f;
      float2 ml = make_float2(-INFINITY, 0.f);
      for (int i = lane; i < n; i += 32) {
        ml = __ldcg(A.cta_ml + at(i) + h);
        if (ml.y != 0.f) M = fmaxf(M, ml.x);
      }
      M = warp_max(M);
      for (int i = lane; i < n; i += 32) {
        if (n > 32) ml = __ldcg(A.cta_ml + at(i) + h);
        const float w = ml.y == 0.f ? 0.f : ml.y * exp2f(ml.x - M) * DOWN<CK>;
        weight[i * S::HG + h] = w;
        sum += w;
      }
      sum = warp_sum(sum);
      if (lane == 0) part_ml[0][h] = make_float2(M, sum);
    }
    __syncthreads();
#pragma unroll 1
    for (int x = 4 * tid; x < hn * HD; x += 4 * THREADS) {
      const int h = x / HD, d = x % HD;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      auto add = [&](int i, float4 v) {
        const float w = weight[i * S::HG + h];
        if (w == 0.f) return;
        acc.x = fmaf(w, v.x, acc.x);
        acc.y = fmaf(w, v.y, acc.y);
        acc.z = fmaf(w, v.z, acc.z);
        acc.w = fmaf(w, v.w, acc.w);
      };
      int i0 = 0;
      if (x == 4 * tid) {
        i0 = FIRST;
#pragma unroll
        for (int i = 0; i < FIRST; ++i)
          if (i < n) add(i, y[i]);
      }
#pragma unroll 8
      for (int i = i0; i < n; ++i) add(i, part(i, x));
      const float M = part_ml[0][h].x, sum = part_ml[0][h].y, inv = sum == 0.f ? 0.f : 1.f / sum;
      const long long head = (long long)p.head * A.group + h0 + h;
      uint16_t* dst = static_cast<uint16_t*>(A.out) + p.seq * A.out_stride + head * HD + d;
      *reinterpret_cast<ushort4*>(dst) = make_ushort4(bits16(acc.x * inv, q_bf16), bits16(acc.y * inv, q_bf16),
                                                      bits16(acc.z * inv, q_bf16), bits16(acc.w * inv, q_bf16));
      if (A.lse && d == 0)
        A.lse[(long long)p.seq * A.n_heads + head] = sum == 0.f ? -INFINITY : (M + log2f(sum / DOWN<CK>)) * LN2;
    }
    __syncthreads();
  }
}

int sm_count() {
  static const int n = [] {
    int dev = 0, v = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      v = 152;
    return std::min(v, MAX_CTAS);
  }();
  return n;
}

// The workspace: counts of arrivals, parts of warps, parts of CTAs.
struct Carve {
  size_t part_o, cta_o, cta_ml, arrived, total;
};
Carve carve(int hg, int hd) {
  Carve w{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += (bytes + 255) & ~size_t(255);
    return at;
  };
  w.arrived = take(MAX_CTAS * 16);
  const size_t rows = (size_t)MAX_CTAS * 2 * hg;
  w.part_o = take((size_t)MAX_CTAS * WARPS * hg * hd * 4);
  w.cta_o = take(rows * hd * 4);
  w.cta_ml = take(rows * 8);
  w.total = off;
  return w;
}

}  // namespace

size_t paged_attention_workspace(int, int n_heads, int n_kv, int head_dim) {
  return carve(n_heads / n_kv <= 8 ? 8 : 16, head_dim).total;
}

int launch_attention_paged(const KvPool& P, rift_dtype cache, const void* q, rift_dtype dt, long long q_stride, int n_heads,
                           const int* seq_lens, int n_seq, const int* page_table, int max_pages, int window,
                           float scale, void* out, long long out_stride, float* lse, char* ws, cudaStream_t st) {
  const int group = n_heads / P.n_kv, hg = group <= 8 ? 8 : 16, hd = P.head_dim;
  Args A = {};
  A.P = P;
  const unsigned long long es = cache == RIFT_E4M3 ? 1 : 2;
  const unsigned long long strides = (P.page_stride | (unsigned long long)P.row_stride | (unsigned long long)P.head_stride) * es;
  A.unit = 16;
  while (A.unit < (1u << 20) && strides % (2 * A.unit) == 0) A.unit *= 2;
  A.page_u = (uint32_t)(P.page_stride * es / A.unit);
  A.row_u = (uint32_t)(P.row_stride * es / A.unit);
  A.head_u = (uint32_t)(P.head_stride * es / A.unit);
  A.scale_page = (uint32_t)P.n_kv << P.ps_shift;
  A.q = q;
  A.q_stride = q_stride;
  A.n_heads = n_heads;
  A.group = group;
  A.hblocks = (group + hg - 1) / hg;
  A.seq_lens = seq_lens;
  A.n_seq = n_seq;
  A.page_table = page_table;
  A.max_pages = max_pages;
  A.window = window;
  A.scale_log2 = scale * 1.4426950408889634f;
  A.out = out;
  A.out_stride = out_stride;
  A.lse = lse;
  const Carve w = carve(hg, hd);
  A.part_o = reinterpret_cast<float*>(ws + w.part_o);
  A.cta_o = reinterpret_cast<float*>(ws + w.cta_o);
  A.cta_ml = reinterpret_cast<float2*>(ws + w.cta_ml);
  A.arrived = reinterpret_cast<unsigned long long*>(ws + w.arrived);
  A.q_bf16 = dt == RIFT_BF16;
  const int grid = sm_count();
  auto go = [&](auto HD, auto CK, auto NB) -> int {
    constexpr int hd_ = decltype(HD)::value, ck = decltype(CK)::value, nb = decltype(NB)::value;
    using S = Shape<hd_, ck, nb>;
    auto kernel = paged_attn_kernel<hd_, ck, nb>;
    static std::atomic<unsigned long long> raised{0};
    if (raise_smem_limit(raised, kernel, S::SMEM) != cudaSuccess) return -1;
    return launch_ex(kernel, dim3(grid), dim3(THREADS), S::SMEM, st, true, A) == cudaSuccess ? 1 : -1;
  };
  auto by_nb = [&](auto HD, auto CK) {
    return hg == 8 ? go(HD, CK, std::integral_constant<int, 1>()) : go(HD, CK, std::integral_constant<int, 2>());
  };
  auto by_cache = [&](auto HD) {
    if (cache == RIFT_E4M3) return by_nb(HD, std::integral_constant<int, CK_E4M3>());
    if (cache == RIFT_F16) return by_nb(HD, std::integral_constant<int, CK_F16>());
    return by_nb(HD, std::integral_constant<int, CK_BF16>());
  };
  return hd == 128 ? by_cache(std::integral_constant<int, 128>()) : by_cache(std::integral_constant<int, 64>());
}

}  // namespace rift
