"""How the paged attention's keys are dealt to workgroups (la_attend_plan.h, plain C++): a small program forms the items as the kernels do, without a GPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_16760_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>
#include "la_attend_plan.h"
using namespace la;
static int dh, Hkv, Hq, page, blocks;
// The items of rows of these lengths: prints and returns 0 if a row's do not follow each other from its first key to its last, in whole pieces, or there are more than there is room for.
static int whole(const std::vector<int> &rows) {
  const int B = (int)rows.size();
  const AtPlan plan = at_plan(dh, Hkv, page, Hq, blocks, B);
  long long keys = 0, n = 0;
  int longest = 0;
  for (int k : rows) {
    keys += k;
    longest = longest > k ? longest : k;
  }
  auto items = [&](int C) {
    long long c = 0;
    for (int k : rows) c += at_rows_items(k, C);
    return (int)c;
  };
  const int C = plan.target > 0 ? at_cut(B, plan.target, keys, longest, items) : AT_UNCUT;
  for (int b = 0; b < B; ++b) {
    const int c = at_rows_items(rows[b], C);
    long long at = 0;
    for (int i = 0; i < c; ++i) {
      const AtItem it{b, b, rows[b], at_item_keys(rows[b], c), i, 0, c, 0};
      const long long first = (long long)it.index * it.C, end = at_item_end(it);
      if (first != at || first % AT_PIECE || (end <= first && rows[b] > 0)) {
        printf("row %d of %d keys: item %d of %d is %lld .. %lld\n", b, rows[b], i, c, first, end);
        return 0;
      }
      at = end;
    }
    if (at != rows[b]) {
      printf("row %d of %d keys ends at %lld\n", b, rows[b], at);
      return 0;
    }
    n += c;
  }
  if (n > plan.items) printf("%lld items, room for %d\n", n, plan.items);
  return n <= plan.items;
}
int main(int, char **v) {
  dh = atoi(v[2]), Hkv = atoi(v[3]), Hq = atoi(v[4]), page = atoi(v[5]), blocks = atoi(v[6]);
  const long long cap = (long long)blocks * page;
  int good = 0, all = 0;
  if (!strcmp(v[1], "alike")) {  // v[7] rows of every length within v[8] of the table's end, of 2^31 - 128 and of 1
    for (long long end : {cap, 0x7fffff80ll, 1ll})
      for (long long k = end - atoi(v[8]); k <= end + atoi(v[8]); ++k)
        if (k >= 0 && k <= cap) {
          good += whole(std::vector<int>(atoi(v[7]), (int)k));
          ++all;
        }
  } else {  // batches of up to v[7] rows of any lengths up to the table's, most of them short or about a common one
    std::mt19937_64 rng((unsigned)atoi(v[8]));
    for (all = 0; all < atoi(v[9]); ++all) {
      const int B = 1 + (int)(rng() % (unsigned)atoi(v[7]));
      std::vector<int> rows(B);
      const long long common = (long long)((double)cap * exp2(-(double)(rng() % 3000) / 100));
      const unsigned kind = rng() % 4;
      for (int &k : rows) {
        const long long any = (long long)((double)cap * exp2(-(double)(rng() % 3200) / 100));
        const long long x = kind == 0 ? any : kind == 1 ? common : kind == 2 ? common - (long long)(rng() % 300) : rng() % 8 ? common / 50 : common;
        k = (int)(x < 0 ? 0 : x < cap ? x : cap);
      }
      good += whole(rows);
    }
  }
  printf("%d of %d\n", good, all);
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("attend_plan")
    (d / "plan.cpp").write_text("#include <cmath>\n" + PROGRAM)
    exe = str(d / "plan")
    subprocess.run(["g++", "-std=c++17", "-O2", "-fsanitize=undefined", "-fno-sanitize-recover", "-Wall", "-Werror", "-I", CSRC, str(d / "plan.cpp"), "-o", exe], check=True)

    def run(*a):
        lines = subprocess.run([exe, *map(str, a)], check=True, capture_output=True, text=True).stdout.splitlines()
        good, all_ = map(int, lines[-1].split(" of "))
        assert good == all_ > 0, lines[:5]

    return run


@pytest.mark.parametrize("dh,Hkv,Hq,B", [(128, 8, 32, 200), (128, 512, 512, 4), (256, 64, 64, 13), (256, 64, 64, 100), (64, 1, 4, 4000), (8, 1, 1, 1), (256, 1, 3, 2), (128, 8, 8, 33)])
@pytest.mark.parametrize("page,blocks", [(16, (1 << 27) - 1), (1, (1 << 31) - 1), (16, 49), (24, 32), (128, 1000)])
def test_rows_alike(plan, dh, Hkv, Hq, B, page, blocks):
    """Rows of one length each, up to the longest that a table can have: where they are not cut they are one item each, however long."""
    plan("alike", dh, Hkv, Hq, page, blocks, B, 260 if B < 300 else 20)


@pytest.mark.parametrize("dh,Hkv,Hq", [(128, 8, 32), (64, 2, 4), (256, 1, 40), (128, 128, 128), (256, 512, 512)])
@pytest.mark.parametrize("rows", [3, 64, 700])
@pytest.mark.parametrize("page,blocks", [(16, (1 << 27) - 1), (16, 256), (64, 2048)])
def test_batches(plan, dh, Hkv, Hq, rows, page, blocks):
    plan("batches", dh, Hkv, Hq, page, blocks, rows, rows + Hkv, 2000 if rows < 100 else 300)
