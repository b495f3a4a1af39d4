"""The staged tiles of attention with 256 queries a tile: what a step reads from LDS
has to be there, in every wave's part, and a stage is written anew only when every
wave is done with it.  Loads to LDS are in flight until a wave waits for them, and
the waits count: the loop's own source runs here over a model of them, in which a
load lands only when a wait says so (on the card most land long before, so that a
wait that is too loose would not show)."""
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_09800_amd", "csrc")


def many():
    src = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "hbf_chunk.hip")).read())
    at = src.index("struct Many {")
    return src, src[at:src.index("\n};\n", at)]


def function(text, name):
    """Source of the member function `name`, signature and body."""
    at = re.search(r"[^\n]*\b%s\([^;{}]*\{" % name, text)
    depth, end = 1, at.end()
    while depth:
        depth += {"{": 1, "}": -1}.get(text[end], 0)
        end += 1
    return text[at.start():end]


MODEL = r"""
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <deque>
#include <map>
#include <set>
#include <vector>
#define __device__
#define __forceinline__ inline
#define __builtin_amdgcn_sched_group_barrier(...)
using std::min;
using std::max;
struct f32x16 {};
@FILE_CONSTANTS@
struct { struct { const void *dev_k = nullptr, *dev_v = nullptr; } layer; } a;
int64_t from_lane(int64_t v, int) { return v; }
template <int D> int k_at(int, int) { return 0; }
template <int D> int v4_at(int, int) { return 0; }

// One wave; every other one does the same.
bool wrong;
std::deque<int> way;          // tiles of the loads that are in flight, the oldest first
std::map<int, int> landed;    // loads of a tile that this wave has waited for
std::set<int> there;          // tiles that every wave has waited for
std::vector<int> held;        // the tile that a stage holds or waits for
std::set<int> read_since;     // stages read since the last barrier
int staging, loads_a_tile;
#define CHECK(x, ...) do { if (!(x)) { wrong = true; std::printf(__VA_ARGS__); } } while (0)

template <int D> struct Many;
uint32_t stage_bytes;
void to_lds(const void *, uint32_t to) {
  const int at = (int)(to / stage_bytes);
  CHECK(at < (int)held.size(), "stage %d of %d\n", at, (int)held.size());
  if (held[at] != staging) {
    CHECK(!read_since.count(at), "tile %d goes where tile %d may still be read\n", staging, held[at]);
    CHECK(held[at] < 0 || there.count(held[at]), "tile %d goes where tile %d is on its way\n", staging, held[at]);
    held[at] = staging;
  }
  way.push_back(staging);
}
template <int N> void loads_left() {
  while ((int)way.size() > N) {
    landed[way.front()]++;
    way.pop_front();
  }
}
void __syncthreads() {
  for (auto &l : landed)
    if (l.second == loads_a_tile) there.insert(l.first);
  read_since.clear();
}
void reads(int tile) {
  CHECK(held[tile % RING] == tile, "tile %d is read where tile %d is\n", tile, held[tile % RING]);
  CHECK(there.count(tile), "tile %d is read before it is there\n", tile);
  read_since.insert(tile % RING);
}

template <int D> struct Many {
@CONSTANTS@
  struct { uint32_t x0 = 0, x1 = 0; int head = 0; } t;
  const uint32_t lds0 = 0;
  const int lane = 0, w = 0;
  int64_t at = 0;
  int pattern = 0;
  std::set<int> k_read, v_read;
  void find(int) {}
  void place(int) {}
  void load_queries() {}
  void nothing_pending() {}
  void add_values() {}
  void probabilities(const f32x16 &, int) {}
  void scores(f32x16 &) {}
  void mask(f32x16 &, uint32_t) {}
  template <bool PENDING> void maximum(const f32x16 &) {}
  bool whole(int i) { return pattern == 2 ? i % 3 == 1 : pattern; }
  void look(int tile) { reads(tile); }
  // (what is read ahead of the last step is not used)
  void read_k(int tile, int first) { if (tile * MANY_TILE < (int)t.x1) { reads(tile); k_read.insert(tile * MANY_TILE + first); } }
  void read_v(int tile, int first) { reads(tile); v_read.insert(tile * MANY_TILE + first); }
@STAGE@
  void stage(int tile) { staging = tile; from_source(tile); }
@REST@
};

template <int D> void replay(int n, int pattern) {
  Many<D> m;
  m.t.x1 = n * MANY_TILE;
  m.pattern = pattern;
  stage_bytes = 2 * Many<D>::TILE_BYTES;
  loads_a_tile = 2 * Many<D>::PASSES;
  way.clear(), landed.clear(), there.clear(), read_since.clear();
  held.assign(RING, -1);
  const bool before = wrong;
  m.run();
  CHECK(way.empty(), "loads are on their way at the end\n");
  for (int x = 0; x < n * MANY_TILE; x += HALF)
    CHECK(m.k_read.count(x) && m.v_read.count(x), "tokens %d .. are not read\n", x);
  if (wrong && !before) std::printf("first of %d tiles, D = %d\n", n, D);
}
int main() {
  for (int pattern = 0; pattern < 3; pattern++)
    for (int n = 1; n <= 40; n++) {
      replay<64>(n, pattern);
      replay<128>(n, pattern);
    }
  return wrong;
}
"""


def replay(tmp_path, change=lambda text: text):
    src, text = many()
    text = change(text)
    file_constants = "\n".join(re.findall(r"^constexpr int (?:MANY_TILE|HALF|RING|MANY_Q|MANY_WAVES)\b[^;]*;", src, re.M))
    constants = "\n".join(re.findall(r"^ *static constexpr int [^;]*;", text, re.M))
    stage = function(text, "stage").replace("void stage(", "void from_source(")
    rest = "\n".join(function(text, f) for f in ("arrived", "step", "run"))
    program = (MODEL.replace("@FILE_CONSTANTS@", file_constants).replace("@CONSTANTS@", constants)
               .replace("@STAGE@", stage).replace("@REST@", rest))
    (tmp_path / "ring.cpp").write_text(program)
    subprocess.run(["g++", "-std=c++17", "-O1", "-w", str(tmp_path / "ring.cpp"), "-o", str(tmp_path / "ring")], check=True)
    return subprocess.run([str(tmp_path / "ring")], capture_output=True, text=True)


def test_tiles_are_there_when_they_are_read(tmp_path):
    r = replay(tmp_path)
    assert r.returncode == 0, r.stdout[-2000:]


@pytest.mark.parametrize("name", ["read_k", "read_v", "look"])
def test_reads_are_of_the_stage_that_the_model_takes(name):
    assert re.search(r"const char \*[kv]t = lds \+ tile % RING \* 2 \* TILE_BYTES( \+ TILE_BYTES)?;", function(many()[1], name))


@pytest.mark.parametrize("is_now,planted", [
    (r"arrived\(min\(n - 2 - i, 1\)\);", "arrived(min(n - 2 - i, 2));"),              # one tile more on its way
    (r"arrived\(min\(n, RING - 1\) - 1\);", "arrived(min(n, RING - 1));"),
    (r"loads_left<N>\(\)", "loads_left<N + 1>()"),                                     # one load more
    (r"if \(i \+ RING - 1 < n\) stage\(i \+ RING - 1\);", "if (i + RING < n) stage(i + RING);"),
    (r"\n\s*__syncthreads\(\);\n", "\n"),                                              # a wave waits for its own alone
])
def test_the_model_finds_what_is_planted(tmp_path, is_now, planted):
    def change(text):
        text, n = re.subn(is_now, planted, text)
        assert n
        return text
    assert replay(tmp_path, change).returncode == 1
