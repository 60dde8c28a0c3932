"""How the paged attention's line is cut, compiled for the host from the kernel's source: the plan that every CTA makes from
the row counts, for short heads and for the longest that a descriptor allows, without a sum past 32 bits."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

MAIN = """
#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdint>
#include <cstdio>
#include <random>
#include <vector>
#define __device__
#define __host__
#define __forceinline__ inline
using std::min;
using std::max;
struct float2 { float x, y; };
struct Cache { int page_shift, max_pages; };
struct { int x; } gridDim;
static int __reduce_add_sync(unsigned, int x) { return x; }
static unsigned __reduce_add_sync(unsigned, unsigned x) { return x; }
%s
// what the kernel sums over the heads, 32 heads a segment and then the segments
template <class S>
static int check(const std::vector<int>& lens, int subs, int ctas, int own) {
  // (the host launches as many CTAs as the longest head that the table allows has tiles, and no more than fit the device)
  const int tallest = *std::max_element(lens.begin(), lens.end());
  const int grid = (int)std::min<long long>(ctas, std::max(1ll, (long long)(tallest + S::kTile - 1) / S::kTile * (long long)lens.size() * subs));
  PageParams p = {};
  p.heads = (int)lens.size();
  p.subs = subs;
  p.own_queries = own;
  p.sms = ctas / 2;
  gridDim.x = grid;
  Counts all = {};
  int most = 0;
  const auto add = [](Counts& a, const Counts& b) {
    a.boxes += b.boxes;
    for (int i = 0; i < kSizes / 2; ++i) a.pieces[i] += b.pieces[i];
  };
  for (size_t h = 0; h < lens.size(); h += 32) {
    Counts seg = {};
    for (size_t i = h; i < std::min(lens.size(), h + 32); ++i) {
      add(seg, Counts::of<S>(lens[i]));
      most = std::max(most, boxes_of(lens[i]));
    }
    add(all, seg.over_warp());
  }
  all = all.over_warp();
  const Plan plan = plan_of<S>(p, all, most);
  long long boxes = 0, longest = 0;
  for (int n : lens) {
    boxes += (n + 15) / 16;
    longest = std::max(longest, (n + 15) / 16 * 1ll);
  }
  if (plan.total != boxes * subs) return 1;
  if (plan.parts < 0 || plan.parts > grid) return 2;
  if (plan.by_warp) return subs == 1 && own && longest * grid * kConsumers <= 2 * boxes ? 0 : 3;
  if (plan.piece) {
    long long n = 0;  // pieces of that size
    const long long tiles = 1ll << (S::kPieceLog + plan.piece - 1);
    for (int len : lens) n += (((len + S::kTile - 1) / S::kTile) + tiles - 1) / tiles;
    if (n * subs != plan.parts) return 4;
    // the smallest sizes are passed over only where every portion is one piece of the third
    const bool whole = longest * 2 * S::kBoxBytes <= 192 * 1024;
    if (plan.piece == 3 && whole && plan.parts != (long long)subs * std::count_if(lens.begin(), lens.end(), [](int x) { return x > 0; }))
      return 5;
    return 0;
  }
  for (int i = 0; i < plan.parts; ++i)  // equal parts: the line from end to end, a tile in each at least
    if (part_begin(plan.total, plan.parts, i + 1) - part_begin(plan.total, plan.parts, i) < std::min(plan.total, kBoxesOf<S>)) return 6;
  if (plan.parts && (part_begin(plan.total, plan.parts, 0) != 0 || part_begin(plan.total, plan.parts, plan.parts) != plan.total)) return 7;
  for (int i = 0; i < plan.parts; ++i)
    if (part_of(plan.total, plan.parts, part_begin(plan.total, plan.parts, i)) != i) return 8;
  return 0;
}
template <class S>
static int all_of(const char* name) {
  std::mt19937 g(7);
  for (int round = 0; round < 3000; ++round) {
    const int heads = 1 << g() %% 13, subs = g() %% 4 ? 1 : 1 + g() %% 3;
    const double scale = std::pow(2.0, g() %% 24);
    std::vector<int> lens(heads);
    long long rows = 0;
    for (int& n : lens) {
      n = g() %% 6 ? (int)std::min((1 << 30) - 1.0, scale * (g() %% 1000) / 1000) : 0;
      rows += (n + 15) / 16 * 16;
    }
    if (rows * subs >= 1ll << 35) continue;  // (the host refuses such calls)
    const int why = check<S>(lens, subs, round %% 5 ? 296 : 2 + 2 * (g() %% 148), g() %% 2);
    if (why) { printf("%%s: %%d heads of up to %%g rows, %%d portions: %%d\\n", name, heads, scale, subs, why); return 1; }
  }
  // the longest heads of all
  for (int n : {1 << 21, (1 << 21) + 1, 1 << 22, 1 << 25, 1 << 27, (1 << 30) - 256})
    for (int heads : {1, 2, 31})
      if (check<S>(std::vector<int>(heads, n), 1, 296, 1)) { printf("%%s: %%d of %%d rows\\n", name, heads, n); return 1; }
  return 0;
}
int main() {
  if (all_of<Shape<128, true, 8>>("bf16 128") | all_of<Shape<128, true, 16>>("bf16 128, 16") | all_of<Shape<64, true, 8>>("bf16 64") |
      all_of<Shape<128, false, 8>>("fp32 128") | all_of<Shape<64, false, 4>>("fp32 64")) return 1;
  puts("cut");
}
"""


def _source():
    text = open(os.path.join(ROOT, "paper_2509_09754_b200", "csrc", "decode_pages.cu")).read()

    def between(first, last):
        i = text.index(first)
        return text[i: text.index(last, i)]

    parts = ["\n".join(re.findall(r"^constexpr int k(?:Consumers|BoxRows) = .*$", text, re.M)),
             between("template <int D, bool BF16, int Q>\nstruct Shape {", "struct Ctl {"),
             between("template <class S>\n__device__ __forceinline__ int tiles_of", "__device__ __forceinline__ int head_len"),
             between("template <class S>\nconstexpr int kBoxesOf", "// A CTA's part:")]
    return "\n".join(parts)


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host compiler")
def test_the_plan_of_the_cut(tmp_path):
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(MAIN % _source())
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", str(src), "-o", str(exe)],
                   check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "cut", r.stdout + r.stderr
