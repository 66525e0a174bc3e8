"""How the trees' attention is shared out (la_tree_plan.h, plain C++): a small program forms items and records as the kernels do, without a GPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_16760_amd", "csrc")

PROGRAM = r"""
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>
#include "la_tree_plan.h"
using namespace la;
static la_pages_desc p;
static int Hq;
// Requests of these keys (0: no rows): 0 if a request's items do not follow each other in whole pieces from its first key to its last, there are more items or records than room, the workspace's
// parts overlap or pass its end, or a model's scratch memory does not hold it.
static int whole(const std::vector<int> &keys, int blocks, int rows) {
  const int R = (int)keys.size();
  const TreePlan plan = ta_plan(p, Hq, blocks, R, rows);
  const size_t record = (size_t)Hq * rows * (p.head_dim + 4) * 4;
  long long all = 0, n = 0, records = 0;
  int longest = 0;
  for (int k : keys) {
    all += k;
    longest = longest > k ? longest : k;
  }
  auto items = [&](int C) {
    long long c = 0;
    for (int k : keys) c += at_rows_items(k, C);
    return (int)c;
  };
  const int C = plan.target > 0 && longest > plan.uncut ? at_cut(R, plan.target, all, longest, items) : AT_UNCUT;
  for (int r = 0; r < R; ++r) {
    const int c = at_rows_items(keys[r], C);
    long long at = 0;
    for (int i = 0; i < c; ++i) {
      const AtItem it{r, r, keys[r], at_item_keys(keys[r], c), i, 0, c, 0};
      const long long first = (long long)it.index * it.C, end = at_item_end(it);
      if (first != at || first % AT_PIECE || (end <= first && keys[r] > 0)) return printf("request %d of %d keys: item %d of %d is %lld .. %lld\n", r, keys[r], i, c, first, end), 0;
      at = end;
    }
    if (at != keys[r]) return printf("request %d of %d keys ends at %lld\n", r, keys[r], at), 0;
    n += c;
    records += c > 1 ? c : 0;
  }
  const size_t room = plan.target > 0 ? plan.notes : 0, list = plan.list ? plan.items * sizeof(AtItem) + (size_t)R * 4 : 0, front = plan.list ? plan.list : plan.bytes;
  if (n > plan.items) return printf("%lld items, room for %d\n", n, plan.items), 0;
  if (records * record > room) return printf("%lld records of %zu bytes, room for %zu\n", records, record, room), 0;
  if (plan.target > 0 ? front < plan.notes + R * TA_NOTE || plan.notes % 16 || front % 16 || (R > 64) != (plan.list > 0) || front + list > plan.bytes : plan.bytes != 0)
    return printf("notes at %zu, list at %zu, %zu bytes\n", plan.notes, plan.list, plan.bytes), 0;
  if (room > TA_RECORDS && plan.target > 1) return printf("records of %zu bytes\n", room), 0;
  if (plan.tiles * (plan.wide ? plan.wide : 16) < Hq / p.n_kv_heads * rows) return printf("%d tiles of %d rows\n", plan.tiles, rows), 0;
  const long long groups = (long long)plan.items * p.n_kv_heads;
  if (plan.grid < 1u << 24 && plan.grid < groups * plan.tiles) return printf("%u workgroups for %lld of %d tiles\n", plan.grid, groups, plan.tiles), 0;
  if (R <= LA_MAX_ROWS && plan.bytes > std::max((size_t)256, tree_attend_bytes(p, Hq))) return printf("%zu bytes, a model has %zu\n", plan.bytes, tree_attend_bytes(p, Hq)), 0;
  return 1;
}
int main(int, char **v) {
  p = la_pages_desc{};
  p.dtype = atoi(v[1]), p.head_dim = atoi(v[2]), p.n_kv_heads = atoi(v[3]), Hq = atoi(v[4]), p.page_size = atoi(v[5]), p.n_layers = 1, p.n_pages = 1;
  const int most = atoi(v[6]), n = atoi(v[7]);
  std::mt19937_64 rng((unsigned)(p.head_dim + most));
  int good = 0, all = 0;
  for (; all < n; ++all) {
    // any number of requests and rows, tables of any length (their number of positions has 31 bits), lengths of any kind up to the table's
    const int R = 1 + (int)(rng() % (unsigned)most), rows = rng() % 3 ? 1 + (int)(rng() % 64) : 1 << rng() % 7;
    const long long positions = (long long)exp2((double)(rng() % 3100) / 100), cap = std::max(1ll, positions / p.page_size) * p.page_size, common = (long long)((double)cap * exp2(-(double)(rng() % 1000) / 100));
    const unsigned kind = rng() % 5;
    std::vector<int> keys(R);
    for (int &k : keys) {
      const long long any = (long long)((double)cap * exp2(-(double)(rng() % 3100) / 100));
      const long long x = kind == 0 ? any : kind == 1 ? cap : kind == 2 ? common - (long long)(rng() % 300) : kind == 3 ? (rng() % 8 ? common / 50 : common) : rng() % 4 ? 0 : common;
      k = (int)(x < 0 ? 0 : x < cap ? x : cap);
    }
    good += whole(keys, (int)(cap / p.page_size), rows);
  }
  // every number of rows and requests that one call of a model may have, at tables of every length that a rule names and its neighbours
  for (int R = 1; most <= 64 && R <= 64; ++R)
    for (int rows = 1; rows <= 64; ++rows)
      for (long long cap : {256, 384, 768, 1000, 4000, 16000, 65000, 1 << 20, 0x7ffffff0})
        for (int d = -1; d <= 1; ++d) {
          const int blocks = (int)std::max(1ll, std::min(0x7fffffffll / p.page_size, cap / p.page_size + d));
          good += whole(std::vector<int>(R, blocks * p.page_size), blocks, rows);
          ++all;
        }
  printf("%d of %d\n", good, all);
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("tree_plan")
    (d / "plan.cpp").write_text(PROGRAM)
    exe = str(d / "plan")
    subprocess.run(["g++", "-std=c++17", "-O2", "-fsanitize=undefined", "-fno-sanitize-recover", "-Wall", "-Werror", "-I", CSRC, "-I", os.path.join(ROOT, "include"), str(d / "plan.cpp"), "-o", exe],
                   check=True)

    def run(*a):
        lines = subprocess.run([exe, *map(str, a)], check=True, capture_output=True, text=True).stdout.splitlines()
        good, all_ = map(int, lines[-1].split(" of "))
        assert good == all_ > 0, lines[:5]

    return run


@pytest.mark.parametrize("dtype,dh,Hkv,Hq,page", [(1, 128, 8, 32, 16), (2, 128, 8, 32, 24), (0, 64, 2, 4, 24), (2, 256, 1, 16, 16), (1, 128, 1, 128, 16), (1, 64, 8, 8, 64), (1, 96, 2, 24, 8), (0, 256, 4, 4, 1),
                                                  (2, 200, 3, 51, 5), (1, 8, 512, 512, 16), (1, 128, 16, 16, 17)])
@pytest.mark.parametrize("requests", [64, 700])
def test_items_and_records_fit(plan, dtype, dh, Hkv, Hq, page, requests):
    """Requests of any number, rows, lengths and tables, and (of 64 at most) what a model keeps for any of them."""
    plan(dtype, dh, Hkv, Hq, page, requests, 3000 if requests <= 64 else 400)
