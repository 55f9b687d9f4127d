"""The line of work of a paged attention launch (csrc/paged_line.cuh), run on the host from the header itself: the units of a
request's row tiles in closed form, and the pieces that the blocks' shares are made of."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROBE = r"""
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
#include "paged_chunk.cuh"
using namespace dmtd;

// a row tile's units by their definition: one, and the keys that its last row sees
static long long units_of(const PagedCut &K, long long c, int n, int i) {
  const long long keys = c + std::min<long long>(n, (i + 1ll) * K.tile), unit = 1ll << K.lg_unit;
  return 1 + (keys <= 0 ? 0 : (keys + unit - 1) / unit);
}
// the row kernel's cuts for its units of 32 to 128 keys, the chunk kernel's
static PagedCut cut(int kind, int G) { return kind < 3 ? paged_cut(PR_ROWS / G, 5 + kind, 1, INT32_MAX, PR_LEAST) : paged_cut(PC_ROWS / G, PC_LG_TK, 1, INT32_MAX, 2); }

static int sums(int G, int kind) {
  const PagedCut K = cut(kind, G);
  std::mt19937 rng(100 * G + kind);
  long long bad = 0;
  auto check = [&](int n, int keys) {
    PagedRequest r{0, 0, n, keys - n, (n + K.tile - 1) / K.tile};
    long long sum = 0;
    for (int m = 0; m <= r.tiles; ++m) {
      bad += r.units_before(K, m) != sum;
      if (m < r.tiles) {
        bad += r.units(K, m) != units_of(K, r.c, n, m);
        sum += units_of(K, r.c, n, m);
      }
    }
  };
  for (int n = 1; n <= 700; n += 1 + n / 40)
    for (int keys = 0; keys <= 2 * n + 300; keys += 1 + keys / 50) check(n, keys);       // below, at and above the rows
  for (int i = 0; i < 3000; ++i) {
    const int n = 1 + rng() % (i % 2 ? 6000 : 300);
    check(n, rng() % (i % 3 ? n + 1 : 1 << 20));
  }
  check(5000, (1 << 30) - 1);
  printf("%lld\n", bad);
  return 0;
}

// All blocks' pieces of a batch, one after the other: every item's units once, in order, and nothing else.
static int walk(int G, int kind, int nkv, int grid) {
  const PagedCut K = cut(kind, G);
  std::mt19937 rng(1000 * G + 10 * kind + nkv + grid);
  using Share = PagedShare<128, 64>;
  static Share::Shared sh;
  long long bad = 0;
  for (int round = 0; round < 60; ++round) {
    const int B = 1 + rng() % 12;
    std::vector<int> start{0}, lens;
    for (int b = 0; b < B; ++b) {
      const int n = rng() % 4 ? rng() % 40 : rng() % 1500;
      start.push_back(start.back() + n);
      lens.push_back(rng() % 3 ? rng() % (n + 1) : n + rng() % 3000);
    }
    PagedAttentionParams P{};
    P.batch = PagedBatch{start.data(), lens.data(), nullptr, B, 1 << 10, start.back()};
    P.pool.lg_page = 4;
    P.nkv = nkv;
    Share share;
    share.total = 0;
    struct Item { int b, i, kvh; long long units; };
    std::vector<Item> items;
    for (int b = 0; b < B; ++b) {
      const PagedRequest r = paged_request(P.batch, P.pool.lg_page, K, b);
      sh.kept[b][0] = r.row0; sh.kept[b][1] = r.n; sh.kept[b][2] = r.c;
      for (int i = 0; i < r.tiles; ++i)
        for (int h = 0; h < nkv; ++h) items.push_back({b, i, h, units_of(K, r.c, r.n, i)});
      share.total += r.units_before(K, r.tiles) * nkv;
    }
    share.n_blocks = (int)std::min<long long>(grid, (share.total + K.least - 1) / K.least);
    if (!share.n_blocks) continue;
    share.each = share.total / share.n_blocks;
    share.rest = share.total - share.each * share.n_blocks;
    size_t at = 0;                     // the item at hand, and how much of it came
    long long come = 0;
    for (int block = 0; block < share.n_blocks && bad < 10; ++block) {
      share.begin = share.start(block);
      share.end = share.start(block + 1);
      long long v = share.begin, before = 0;
      int b = 0;
      PagedRequest r = share.request(P, K, sh, 0);
      while (v - before >= r.units_before(K, r.tiles) * nkv) {
        before += r.units_before(K, r.tiles) * nkv;
        r = share.request(P, K, sh, ++b);
      }
      PagedPiece p = share.piece_of(P, K, r, v - before);
      for (long long u = share.begin;;) {
        if (at >= items.size()) { ++bad; break; }
        const Item &it = items[at];
        bad += p.r.b != it.b || p.i != it.i || p.kvh != it.kvh || p.t0 != come || p.per_item != it.units || p.t1 <= p.t0 || p.t1 > p.per_item;
        bad += share.holder(u) != block || p.rows(K) < 1 || p.first(K) + p.rows(K) > p.r.n;
        come = p.t1;
        if (come == it.units) { ++at; come = 0; }
        u += p.t1 - p.t0;
        if (bad || !share.next(P, K, sh, p, u)) { bad += u != share.end; break; }
      }
    }
    bad += at != items.size();
  }
  printf("%lld\n", bad);
  return 0;
}

// A share whose end lies behind the line's: its pieces end with the batch's last request all the same.
static int past() {
  const PagedCut K = cut(3, 4);
  static PagedShare<128, 64>::Shared sh;
  long long bad = 0;
  for (int waits = 0; waits < 3; ++waits) {                    // requests without rows at the batch's end
    const int start[4] = {0, 100, waits < 2 ? 300 : 100, waits < 1 ? 301 : start[2]}, lens[3] = {100, 900, 50};
    PagedAttentionParams P{};
    P.batch = PagedBatch{start, lens, nullptr, 3, 1 << 10, start[3]};
    P.pool.lg_page = 4;
    P.nkv = 2;
    int items = 0;
    for (int b = 0; b < 3; ++b) {
      const PagedRequest r = paged_request(P.batch, P.pool.lg_page, K, b);
      sh.kept[b][0] = r.row0; sh.kept[b][1] = r.n; sh.kept[b][2] = r.c;
      items += r.tiles * P.nkv;
    }
    for (int b = 3; b < 64; ++b) sh.kept[b][1] = 7;            // what lies behind the batch
    PagedShare<128, 64> share{};
    share.end = 1 << 20;
    PagedPiece p = share.piece_of(P, K, share.request(P, K, sh, 0), 0);
    long long u = p.t1;
    while (items > 0 && share.next(P, K, sh, p, u)) {
      u += p.t1 - p.t0;
      --items;
    }
    bad += items != 1;
  }
  printf("%lld\n", bad);
  return 0;
}

int main(int argc, char **argv) {
  auto a = [&](int i) { return atoi(argv[i]); };
  if (argc == 1) return past();
  return argc == 3 ? sums(a(1), a(2)) : walk(a(1), a(2), a(3), a(4));
}
"""


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    d = tmp_path_factory.mktemp("probe")
    src, exe = d / "probe.cu", d / "probe"
    src.write_text(PROBE)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-std=c++17", "-O1", "-I",
                    os.path.join(ROOT, "paper_2510_11958_b200", "csrc"), str(src), "-o", str(exe)], check=True)

    def run(*args):
        return int(subprocess.run([str(exe)] + [str(x) for x in args], check=True, capture_output=True, text=True, timeout=300).stdout)
    return run


@pytest.mark.parametrize("kind", [0, 1, 2, 3])
@pytest.mark.parametrize("G", range(1, 17))
def test_units_in_closed_form(probe, G, kind):
    assert probe(G, kind) == 0


@pytest.mark.parametrize("kind", [1, 3])
@pytest.mark.parametrize("G,nkv,grid", [(1, 8, 148), (1, 1, 7), (2, 8, 296), (4, 2, 148), (5, 3, 31), (16, 1, 148)])
def test_shares_hold_every_item_once(probe, G, nkv, grid, kind):
    assert probe(G, kind, nkv, grid) == 0


def test_no_piece_behind_the_last_request(probe):
    assert probe() == 0
