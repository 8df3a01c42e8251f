"""Words of a key mask (cache.h seen_word, seen_words) compiled for the host: the states that they leave, and no word behind the mask's last
or the sequence's end is read."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_no_word_behind_the_mask_or_the_length_is_read(tmp_path):
    if not shutil.which("g++"):
        pytest.skip("g++ not available")
    src = tmp_path / "mask.cpp"
    src.write_text(r'''
#include <cstdio>
#include <vector>
#include "cache.h"
using namespace rs;
int main() {
  uint32_t x = 12345;
  for (int nwords = 1; nwords <= 9; ++nwords)
    for (int total = 0; total <= 32 * nwords; ++total)
      for (int kind = 0; kind < 3; ++kind) {
        std::vector<uint32_t> mask(nwords);
        for (auto &w : mask) w = kind == 0 ? 0u : kind == 1 ? ~0u : (x = x * 1664525u + 1013904223u);
        int last = -1;
        const auto word = [&](int w) {
          last = last > w ? last : w;
          return w >= 0 && w < nwords ? mask[w] : 0u;
        };
        for (int j = 0; j <= 32 * nwords + 96; j += 32) {  // tiles of the kernels reach behind the end
          last = -1;
          const uint32_t got = seen_word(total, j, word);
          if (last >= nwords || (last >= 0 && 32 * last >= total)) return printf("word %d of %d, %d states\n", last, nwords, total), 1;
          for (int i = 0; i < 32; ++i) {
            const uint32_t want = j + i < total ? mask[(j + i) / 32] >> ((j + i) % 32) & 1u : 0u;
            if ((got >> i & 1u) != want) return printf("bit %d of %d\n", j + i, total), 1;
          }
        }
        for (int j = 0; j < total; j += 64) {
          last = -1;
          const uint64_t got = seen_words(total, j, word);
          if (last >= nwords || 32 * last >= total) return printf("word %d of %d, %d states\n", last, nwords, total), 1;
          for (int i = 0; i < 64; ++i) {
            const uint64_t want = j + i < total ? mask[(j + i) / 32] >> ((j + i) % 32) & 1u : 0u;
            if ((got >> i & 1u) != want) return printf("bit %d of %d\n", j + i, total), 1;
          }
        }
      }
  printf("ok\n");
}
''')
    exe = tmp_path / "mask"
    subprocess.run(["g++", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2608_29058_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr
