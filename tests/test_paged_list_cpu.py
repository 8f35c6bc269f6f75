"""The paged attention's list of tiles (functions of the CUDA sources that also compile for the host): quotients, shares,
and the item that each tile and each border belongs to (CPU only; needs nvcc)."""
import random
import subprocess

import pytest

from paper_2609_29029_gb300 import build

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "paged_list.cuh"
// Reads lists (per_seq, n_seq, tiles of each sequence) and prints, for each border of 152 shares (the list's end among them)
// and for each tile of a short list, the item found: x, seq, block, n, base; -1 for a division by zero.
int main() {
  int per_seq, n;
  while (scanf("%d %d", &per_seq, &n) == 2) {
    std::vector<int> t(n);
    std::vector<long long> before(n);
    long long W = 0;
    for (int i = 0; i < n; ++i) {
      if (scanf("%d", &t[i]) != 1) return 1;
      before[i] = W;
      W += t[i];
    }
    W *= per_seq;
    const rift::Shares shares(W, 152);
    auto show = [&](long long x) {
      bool empty = false;
      auto tiles = [&](int i) {
        empty = t[i] == 0;
        return empty ? 1 : t[i];
      };
      const rift::ListItem it = rift::item_at(x, W, per_seq, before.data(), n, tiles);
      printf("%lld %d %d %d %lld %d\n", x, it.seq, it.block, empty ? -1 : it.n, it.base,
             x < W ? shares.owner(x) : 151);
    };
    for (int c = 0; c <= 152; ++c) show(shares.begin(c));
    if (W <= 2000)
      for (long long x = 0; x < W; ++x) show(x);
    printf("end\n");
  }
  // quotients of every size class
  unsigned long long s = 88172645463325252ull;
  for (int k = 0; k < 2000000; ++k) {
    s ^= s << 13; s ^= s >> 7; s ^= s << 17;
    const long long a = (long long)(s >> 1) >> (s % 62);
    s ^= s << 13; s ^= s >> 7; s ^= s << 17;
    const long long b = ((long long)(s >> 1) >> (s % 62)) + 1;
    if (rift::divide(a, b) != a / b) { printf("divide %lld %lld\n", a, b); return 1; }
  }
  return 0;
}
"""


def test_items_and_shares(tmp_path):
    try:
        nvcc = build.nvcc()
    except RuntimeError:
        pytest.skip("no nvcc")
    src, exe = tmp_path / "list.cu", tmp_path / "list"
    src.write_text(PROGRAM)
    subprocess.run([nvcc, "-std=c++17", "-O2", "--expt-relaxed-constexpr", "-I", str(build.ROOT / "include"), "-I",
                    str(build.CSRC), *build.ARCH, str(src), "-o", str(exe)], check=True, capture_output=True)
    rng = random.Random(5)
    lists = [(1, [1]), (1, [7, 0]), (3, [0, 5, 0, 0]), (32, [40] * 5), (8, [0, 0, 300, 0, 1, 0]), (1, [1 << 26] * 40),
             (65536, [1 << 20] * 7 + [0]), (4, [1] * 1024)]
    for _ in range(60):
        n = rng.choice([1, 2, 5, 33, 200])
        t = [rng.choice([0, 0, 1, 2, rng.randrange(1, 60), rng.randrange(1, 5000)]) for _ in range(n)]
        lists.append((rng.choice([1, 2, 8, 33]), t if any(t) else t + [3, 0]))
    text = "".join(f"{p} {len(t)} {' '.join(map(str, t))}\n" for p, t in lists)
    out = subprocess.run([str(exe)], input=text, check=True, capture_output=True, text=True).stdout.split("end\n")[:-1]
    assert len(out) == len(lists)
    for (per_seq, t), block in zip(lists, out):
        W = per_seq * sum(t)
        rows = [[int(x) for x in line.split()] for line in block.splitlines()]
        each, more = divmod(W, 152)
        borders = [each * c + min(c, more) for c in range(153)]
        assert [r[0] for r in rows[:153]] == borders
        before = [0]
        for k in t:
            before.append(before[-1] + per_seq * k)
        for x, seq, blk, n, base, owner in rows:
            tile = min(x, W - 1)
            assert n == t[seq] > 0, (per_seq, t, x)  # a sequence with tiles: no division by zero
            assert 0 <= blk < per_seq and base == before[seq] + blk * n and base <= tile < base + n
            if x < W:
                assert borders[owner] <= x < borders[owner + 1]
