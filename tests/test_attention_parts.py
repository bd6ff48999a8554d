"""How many blocks share a tile of attention: by what the pass streams, not by what it does not."""
import os
import shutil
import subprocess

import pytest

from paper_1910_05124_b200.build import _nvcc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "pm_attn_packed.cuh"
// tokens kv_tokens sequences heads kv_heads rows most least
int main(int, char** s) {
  long v[8];
  for (int i = 0; i < 8; ++i) v[i] = std::atol(s[i + 1]);
  pm::PackedArgs a{};
  a.tokens = v[0]; a.kv_tokens = v[1]; a.n_seqs = (int)v[2]; a.heads = (int)v[3]; a.kv_heads = (int)v[4]; a.group = a.heads / a.kv_heads; a.cross = v[0] != v[1];
  const long forward = pm::most_tiles(a.tokens, a.n_seqs, (int)v[5]) * a.heads;
  const long both = forward + pm::most_tiles(a.kv_tokens, a.n_seqs, (int)v[5]) * a.kv_heads;
  std::printf("%d %d\n", pm::forward_parts(forward, a, (int)v[5], (int)v[6], (int)v[7]), pm::backward_parts(both, a, (int)v[5], (int)v[6], (int)v[7]));
}
"""


@pytest.fixture(scope="module")
def parts(tmp_path_factory):
    if not (os.path.exists(_nvcc()) or shutil.which(_nvcc())):
        pytest.skip("no nvcc")
    at = tmp_path_factory.mktemp("parts")
    (at / "parts.cu").write_text(PROGRAM)
    subprocess.run([_nvcc(), "-std=c++17", "-arch=sm_100a", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_1910_05124_b200", "csrc"),
                    str(at / "parts.cu"), "-o", str(at / "parts")], check=True)

    def run(*values):
        out = subprocess.run([str(at / "parts"), *map(str, values)], capture_output=True, text=True, check=True, timeout=60)
        return tuple(map(int, out.stdout.split()))
    return run


def largest(blocks, streamed, most, least):
    return max(p for p in (1, 2, 4, 8) if p == 1 or blocks * p <= most and streamed >= p * least)


def up(a, b):
    return -(-a // b)


# (rows, most blocks, streamed tiles to a part): tensor cores and CUDA cores
@pytest.mark.parametrize("rows,most,least", [(128, 296, 3), (32, 592, 2), (64, 592, 3)])
@pytest.mark.parametrize("tokens,kv,seqs,heads,kv_heads", [
    (4000, 100, 1, 1, 1), (2000, 40, 1, 2, 2), (1500, 64, 3, 2, 1),                  # long queries over short keys
    (100, 4000, 1, 1, 1), (500, 3000, 1, 2, 2), (60, 1000, 4, 4, 2),                 # and short ones over long keys
    (2000, 2000, 1, 2, 1), (4000, 4000, 1, 4, 4), (1013, 1013, 3, 4, 2)])            # a sequence's own tokens
def test_parts(parts, tokens, kv, seqs, heads, kv_heads, rows, most, least):
    forward, backward = parts(tokens, kv, seqs, heads, kv_heads, rows, most, least)
    q_tiles, k_tiles = (up(up(n, seqs), rows) for n in (tokens, kv))
    blocks, blocks_kv = (tokens // rows + seqs) * heads, (kv // rows + seqs) * kv_heads
    assert forward == largest(blocks, k_tiles, most, least)
    assert backward == largest(blocks + blocks_kv, max(q_tiles * heads // kv_heads, k_tiles), most, least)
    if kv <= 2 * rows:
        assert forward == 1                       # nothing to share out
