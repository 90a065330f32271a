"""The layout of cross attention's plans (host code, compiled here without a GPU): every row meets every key of its source once,
also where list entries end at 2^31 - 1, and lists that no launch can take are refused before they are looked at."""
import os
import subprocess

import pytest

from paper_1702_02181_amd import build_lib as B
from tests.test_oracle_vocab import F, NULL_STREAM  # noqa: F401  (F is a fixture)

MAIN = r'''
#include <cstdio>
#include <map>
#include <set>
#include "cross_plan.hip"
using namespace fold;
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
typedef std::pair<int64_t, int64_t> Part;

// spans that follow each other from begin to end
static bool whole(std::vector<Part> v, int64_t begin, int64_t end) {
  std::sort(v.begin(), v.end());
  for (const Part& s : v) {
    if (s.first != begin || s.second < s.first) return false;
    begin = s.second;
  }
  return begin == end;
}

static int check(const std::vector<int32_t>& qp, const std::vector<int32_t>& kp, const std::vector<int32_t>& src, int G, int kv,
                 int least) {
  const int64_t sources = (int64_t)kp.size() - 1;
  Lists l{qp, kp, G, kv, least, {}, {}};
  l.first.push_back(0);
  for (int64_t e = 0; e <= sources; ++e) {
    for (int s = 0; s < (int)src.size(); ++s)
      if (src[s] == e || (src[s] < 0 && e == sources)) l.seqs.push_back(s);
    l.first.push_back((int32_t)l.seqs.size());
  }
  for (int height : {32, 128}) {
    std::vector<QTile> tiles, join;
    int slots = 0;
    query_tiles(l, height, &tiles, &join, &slots);
    CHECK(tiles.size() % 8 == 0);
    std::map<std::pair<int, int>, std::vector<Part>> keys;  // by (entry, head within the group): spans of keys
    std::set<int> used;
    for (const QTile& t : tiles) {
      if (t.rows == 0) continue;
      CHECK(t.rows <= height && (t.slot < 0 || used.insert(t.slot).second) && t.slot < slots);
      for (int r = 0; r < t.rows; ++r) keys[{t.entry + (t.head0 + r) / G, (t.head0 + r) % G}].push_back({t.k_begin, t.k_end});
    }
    for (size_t s = 0; s < src.size(); ++s)
      for (int64_t i = qp[s]; i < qp[s + 1]; ++i)
        for (int g = 0; g < G; ++g) {
          const auto& v = keys[{(int)i, g}];
          if (src[s] < 0 || kp[src[s]] == kp[src[s] + 1]) CHECK(v.size() == 1 && v[0].first == v[0].second);
          else CHECK(whole(v, kp[src[s]], kp[src[s] + 1]));
          keys.erase({(int)i, g});
        }
    CHECK(keys.empty());
    size_t pieces = 0;
    for (const QTile& t : join) pieces += t.pieces;
    CHECK((int)pieces == slots);
  }
  for (int height : {32, 64}) {
    std::vector<KTile> tiles, join;
    std::vector<RTile> rows;
    int slots = 0;
    key_tiles(l, height, &tiles, &join, &rows, &slots);
    std::map<int64_t, std::vector<Part>> runs;  // by first key: spans of row tiles
    std::map<int64_t, int64_t> end;
    for (const KTile& t : tiles) {
      if (t.keys == 0) continue;
      CHECK(t.keys > 0 && t.keys <= kCrossKeys && (int64_t)t.k_begin + t.keys <= INT32_MAX);
      runs[t.k_begin].push_back({t.t_begin, t.t_end});
      end[t.k_begin] = (int64_t)t.k_begin + t.keys;
    }
    int64_t row = 0;
    for (int64_t e = 0; e < sources; ++e) {
      int64_t n = 0;
      for (int s : l.readers(e)) n += (((int64_t)qp[s + 1] - qp[s]) * G + height - 1) / height;
      for (int64_t k = kp[e]; k < kp[e + 1]; k = end[k]) {
        CHECK(end.count(k) && end[k] <= kp[e + 1] && whole(runs[k], row, row + n));
        runs.erase(k);
      }
      row += n;
    }
    CHECK(runs.empty() && row == (int64_t)rows.size());
  }
  // rows of sources with up to `most` keys in tiles, other rows that read a key listed, each once
  for (int most : {1, 32, 100}) {
    std::vector<QTile> tiles;
    std::vector<int32_t> others;
    brief_tiles(l, most, &tiles, &others);
    std::map<int64_t, int64_t> source;
    for (size_t s = 0; s < src.size(); ++s)
      for (int64_t i = qp[s]; i < qp[s + 1]; ++i)
        if (src[s] >= 0 && kp[src[s]] < kp[src[s] + 1]) source[i] = src[s];
    for (int32_t i : others) CHECK(source.count(i) && kp[source[i] + 1] - kp[source[i]] > most && source.erase(i));
    std::set<std::pair<int64_t, int>> seen;
    for (const QTile& t : tiles)
      for (int r = 0; r < t.rows; ++r) {
        const int64_t i = t.entry + (t.head0 + r) / G;
        CHECK(source.count(i) && t.k_begin == kp[source[i]] && t.k_end == kp[source[i] + 1] && t.k_end - t.k_begin <= most);
        CHECK(t.rows <= kCrossBriefRows && t.slot == -1 && seen.insert({i, (t.head0 + r) % G}).second);
      }
    CHECK(seen.size() == source.size() * G);
  }
  return 0;
}

int main() {
  const int32_t top = INT32_MAX;  // past the last entry that a plan takes
  if (check({0, 5, 5, 300}, {0, 70, 70, 1000}, {0, 1, 2}, 1, 1, 128)) return 1;
  if (check({0, 1, 2, 3, 260}, {0, 130, 9000}, {1, 1, -1, 0}, 3, 2, 256)) return 1;
  if (check({0, 9, 700, 701, 720, 730}, {0, 1, 33, 33, 66}, {3, 1, 0, 2, 1}, 4, 2, 256)) return 1;
  if (check({0, 700}, {top - 5000, top - 4999, top}, {1}, 2, 1, 128)) return 1;
  if (check({0, 700, 701}, {top - 100, top}, {0, 0}, 1, 4, 256)) return 1;
  if (check({top - 300, top - 1, top}, {0, 2000}, {0, 0}, 1, 1, 128)) return 1;
  std::printf("fine\n");
  return 0;
}
'''


def test_layout(tmp_path):
    (tmp_path / "main.hip").write_text(MAIN)
    r = subprocess.run([B.HIPCC, "-x", "hip", "--offload-host-only", "-std=c++17", "-O1", "-ftrapv", "-I" + B.CSRC,
                        "-I" + os.path.join(B.ROOT, "include"), str(tmp_path / "main.hip"),
                        "-Wl,--unresolved-symbols=ignore-all", "-o", str(tmp_path / "layout")],
                       capture_output=True, text=True)  # (the device code is left out)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout == "fine\n", (r.returncode, r.stdout)


@pytest.mark.parametrize("kw", [dict(num_keys=2 ** 31 - 1, num_key_rows=2 ** 31 - 1),
                                dict(num_keys=2 ** 31 - 1151, num_key_rows=2 ** 31 - 1),
                                dict(num_queries=2 ** 31 - 1, num_query_rows=2 ** 31 - 1),
                                dict(heads=64, num_queries=2 ** 25 - 1, num_query_rows=2 ** 25)])
def test_too_many_tiles_are_refused_unseen(F, kw):  # noqa: F811
    ok = dict(dtype=0, heads=1, kv_heads=1, head_dim=64, num_seqs=1, num_sources=1, num_queries=10, num_keys=20,
              num_query_rows=10, num_key_rows=20, query_ptr=4096, query_row=None, key_ptr=8192, key_row=None, source=None)
    with pytest.raises(F.FoldError, match="too many tiles") as e:
        F.fold_cross_create(F.fold_cross_batch(**dict(ok, **kw)), NULL_STREAM)
    assert e.value.code == F.FOLD_E_INVALID
