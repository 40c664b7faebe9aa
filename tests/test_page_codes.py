"""CPU: the quotient that gr_page_write makes of a scale's reciprocal and one correction is the division's."""
import subprocess

SOURCE = r"""
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>
static float bits(uint32_t u) { float x; memcpy(&x, &u, 4); return x; }
int main(void) {
#ifdef __FMA__
  const uint32_t every = 1;
#else
  const uint32_t every = 61;          /* fused products in software: some of the scales */
#endif
  long other = 0, plain = 0;
  for (uint32_t m = 0; m < 1u << 23; m += every) {
    const float s = bits(0x3f800000u | m), r = 1.0f / s;
    for (uint32_t k = 0; k < 128; k++) {
      const float x = bits(0x3f800000u | k << 16), q0 = x * r;
      other += fmaf(fmaf(-q0, s, x), r, q0) != x / s;
      plain += q0 != x / s;
    }
  }
  printf("%ld %d\n", other, plain > 0);
  return 0;
}
"""


def test_corrected_reciprocal_for_all_significands(tmp_path):
    """Of all 2^23 significands of a scale and all 128 of a bf16 value none gives another quotient (a product with the reciprocal alone does)."""
    (tmp_path / "q.c").write_text(SOURCE)
    subprocess.run(["gcc", "-O3", "-march=native", "-ffp-contract=off", "q.c", "-o", "q", "-lm"], cwd=tmp_path, check=True)
    assert subprocess.run(["./q"], cwd=tmp_path, check=True, capture_output=True, text=True).stdout.split() == ["0", "1"]
