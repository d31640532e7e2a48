"""Which scale bytes the 8-bit product asks for (no GPU: the kernels' own arithmetic, compiled for the host).

The kernels that walk k in stages hold the scale words of whole groups of stages and ask for a group at a time, as far as
past the end of a row.  What lies past the last row is not the operand's: no byte from there on may be asked for."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2508_17588_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

PROGRAM = r'''
#include "%s/hero_kernels.h"
#include <cstdio>
int main() {
  long bad = 0;
  for (int k = 16; k <= 1 << 17; k += k < 4096 ? 16 : 1008) {
    const int pitch = fp8_scale_pitch(k), stages = (k + 127) / 128;
    for (int stage = 0; stage < stages; stage += 4)                 // groups and chunks begin on whole words
      for (int w = 0; w < 16; ++w) {
        const int at = fp8_scale_word_offset(stage / 4 + w, pitch);
        const bool used = stage + 4 * w < stages;
        if (at < 0 || at + 4 > pitch || (used && at != stage + 4 * w)) {
          if (bad++ == 0) printf("k %%d stage %%d word %%d: byte %%d of %%d\n", k, stage, w, at, pitch);
        }
      }
  }
  return bad != 0;
}
'''


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_scale_words_stay_within_their_row(tmp_path):
    src, exe = tmp_path / "words.hip", tmp_path / "words"
    src.write_text(PROGRAM % CSRC)
    res = subprocess.run([HIPCC, "--offload-arch=gfx950", "-std=c++17", "-O0", str(src), "-o", str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    res = subprocess.run([str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout


def test_every_scale_load_with_a_scalar_offset_is_limited():
    text = open(os.path.join(CSRC, "gemm_fp8.hip")).read()
    loads = re.findall(r"raw_buffer_load_b32\(rsSA,([^;]*), 0\);", text)
    assert len(loads) == 3, loads
    for load in loads:
        offset = load.rsplit(",", 1)[1].strip() if "fp8_scale_word_offset" not in load else "fp8_scale_word_offset"
        assert offset in ("word", "fp8_scale_word_offset"), load
    assert "const int word = fp8_scale_word_offset(stage / 4 + w, pitch);" in text
    # scales brought straight into LDS: the whole advance lies in the checked offset
    for fill in re.findall(r"lds_fill\(rsS[AW],[^;]*;", text):
        assert fill.count(",") == 2, fill
