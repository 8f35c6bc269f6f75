// The list of tiles that the paged attention works off: items (sequence, block of heads) one after the other, each with
// the tiles of its sequence.  Which item a tile belongs to, and how the list is cut into shares.
#pragma once

#include "rift_common.cuh"

namespace rift {

// a / b for a >= 0, b > 0.  Three cases by size, as a 64-bit division takes hundreds of cycles and a 32-bit one about a
// hundred: quotients below 2^20 by fp32 (off by one at most, put right).
// (Not inlined: a small call runs each instruction about once, and fetching them is most of its time.)
__host__ __device__ __noinline__ inline long long divide(long long a, long long b) {
  if (((a | b) >> 31) != 0) return a / b;
  const int x = (int)a, y = (int)b;
#ifdef __CUDA_ARCH__
  const float f = __fdividef((float)x, (float)y);
#else
  const float f = (float)x / (float)y;
#endif
  if (f >= 1048576.f) return (uint32_t)x / (uint32_t)y;
  int q = (int)f, r = x - q * y;
  if (r < 0) --q;
  else if (r >= y) ++q;
  return q;
}
// n things cut into k shares, the first ones a thing larger.
struct Shares {
  long long each, more;
  __host__ __device__ __forceinline__ Shares(long long n, int k) : each(divide(n, k)), more(n - each * k) {}
  __host__ __device__ __forceinline__ long long begin(int i) const { return each * i + (i < more ? i : more); }
  __host__ __device__ __forceinline__ int owner(long long x) const {  // the share that holds thing x
    const long long large = more * (each + 1);
    return (int)(x < large ? divide(x, each + 1) : more + divide(x - large, each));
  }
};

// The item that holds tile x of a list of W > 0 tiles, for 0 <= x < W; the last one for x = W (a border behind the list:
// sequences without tiles may follow the last item, and have no item to find).  Each sequence has per_seq items of tiles(i)
// tiles; before[i] is the tiles of an item of each sequence before i.
struct ListItem {
  int seq, block, n;  // block: which of the sequence's items; n: its tiles
  long long base;     // tiles of the items before it
};
template <typename Tiles>
__host__ __device__ __forceinline__ ListItem item_at(long long x, long long W, int per_seq, const long long* before, int n_seq,
                                                     Tiles tiles) {
  if (x >= W) x = W - 1;
  const long long want = divide(x, per_seq);
  int lo = 0, hi = n_seq;  // the last sequence with `want` tiles or fewer before it
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (before[mid] <= want) lo = mid;
    else hi = mid;
  }
  ListItem it;
  it.seq = lo;
  it.n = tiles(lo);
  it.base = before[lo] * per_seq;
  it.block = (int)divide(x - it.base, it.n);
  it.base += (long long)it.block * it.n;
  return it;
}

}  // namespace rift
