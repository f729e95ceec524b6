"""How the rotating kernel's blocks number their items (csrc/move_cut.cuh), gone over on the CPU: every item of every block is one
piece of one head of one token, no two the same."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2306_14048_b200", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <initializer_list>
#include "move_cut.cuh"
static bool sound(int64_t n_tokens, int heads, int per, int half) {
  int64_t parts;
  const h2o::MoveCut cut = h2o::move_cut(n_tokens, heads, per, half, 148, parts);
  bool ok = cut.tokens >= 1 && cut.tokens <= h2o::kMaxTokens && cut.items == heads * per && cut.tokens * half <= h2o::kMaxHalf && parts >= 1;
  for (int i = 0; ok && i < cut.items * cut.tokens; ++i) {
    int token, head, c;
    cut.split(i, token, head, c);
    ok = token >= 0 && token < cut.tokens && head >= 0 && head < heads && c >= 0 && c < per && (token * heads + head) * per + c == i;
  }
  if (!ok) printf("%lld tokens, %d heads, %d items of a head, %d pairs: %d tokens to a block\n", (long long)n_tokens, heads, per, half, cut.tokens);
  return ok;
}
int main() {
  int bad = 0;
  const int64_t counts[] = {1, 7, 1184, 1185, 5000, 100000};
  for (int64_t n : counts)
    for (int dim = 8; dim <= 512; dim += 8)
      for (int wide = 4; wide <= 8; wide += 4)  // values of 16 bytes
        for (int pairs = 0; pairs < 3; ++pairs) {  // one pair to an item, or two chunks
          if (pairs == 0 && dim % (2 * wide) != 0) continue;
          const int per = pairs == 0 ? dim / (2 * wide) : dim / 2;
          const int half = pairs == 2 ? 1 : dim / 2;
          for (int heads = 1; heads <= 40; heads += heads < 6 ? 1 : 17) bad += !sound(n, heads, per, half);
        }
  for (int heads : {65535, 3 * 65535}) bad += !sound(3, heads, 64, 64);
  bad += !sound(3, 65535, 256, 256);  // the most heads of the most channels
  return bad != 0;
}
"""


def test_every_item_is_one_piece_of_one_head(tmp_path):
    source, program = tmp_path / "cut.cpp", str(tmp_path / "cut")
    source.write_text(PROGRAM)
    subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-x", "c++", "-I", CSRC, str(source), "-o", program], check=True)
    res = subprocess.run([program], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, res.stdout[:2000]
