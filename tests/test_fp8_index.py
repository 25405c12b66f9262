"""The FP8 kernels' index arithmetic at the largest sizes, compiled for the host with overflow checks."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2307_09782_b200", "csrc")
MOST_ROWS = 0x7FFFFF00  # what the entry points accept


def run(tmp_path, body):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text('#include <cstdint>\n#include <cstdio>\n#include "fp8_index.h"\nusing namespace zq::fp8b;\nint main() {\n' + body +
                   "\nreturn 0; }\n")
    subprocess.run(["g++", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", CSRC, str(src), "-o", str(exe)],
                   check=True)
    return subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout


def test_weight_gradient_rows(tmp_path):
    """Every token that a converter reads a scale of exists, for all its stages and those it looks ahead to, with the tokens
    shared by 1 - 8 CTAs; and every token is read.  (Past the last stage a token number beyond 2^31 turned negative and passed
    for one inside.)"""
    body = """
  const int sizes[] = {1, 63, 64, 65, 4097, 0x7FFFFEC1, 0x7FFFFEFF, 0x7FFFFF00};
  for (int M : sizes)
    for (int cluster = 1; cluster <= 8; cluster *= 2) {
      const int all = static_cast<int>((static_cast<int64_t>(M) + 63) / 64);
      for (int rank = 0; rank < cluster; ++rank) {
        const int step0 = static_cast<int>(static_cast<int64_t>(all) * rank / cluster);
        const int steps = static_cast<int>(static_cast<int64_t>(all) * (rank + 1) / cluster) - step0;
        for (int i = steps > 8 ? steps - 8 : 0; i < steps + 8; ++i)
          for (int row = 0; row < 64; ++row) {
            const int m = stage_token(step0, i, steps, row, M);
            const int64_t want = (static_cast<int64_t>(step0) + i) * 64 + row;
            if (m != (i < steps && want < M ? want : -1)) return 1;
          }
      }
    }"""
    run(tmp_path, body)


def test_chained_kernels_load_through_l2():
    """The kernels that are launched before the one ahead has ended never use the read-only path, whose loads may see what was
    there before (and may be moved ahead of the wait)."""
    for name in ("fp8_block_few.cu", "fp8_block_gemm.cu", "fp8_wgrad.cu"):
        text = open(os.path.join(CSRC, name)).read()
        assert "__ldg(" not in text and "__restrict__" not in text and "load_chained(" in text, name
    text = open(os.path.join(CSRC, "fp8_block_quant.cu")).read()
    chained = text[text.index("\nquantize_block_kernel("):text.index("// One CTA per 128 x 128 block")]
    assert "__ldg(" not in chained and "__restrict__" not in chained and "pdl_wait();" in chained


def test_row_bytes(tmp_path):
    """Rows of up to 2^31 elements: whole pieces as long as there are enough left (their bytes, counted first, overflowed from
    2^29 elements of four bytes on, and nothing was stored)."""
    body = """
  const int lefts[] = {0, 1, 31, 32, 33, 63, 64, 65, 1 << 28, 1 << 29, (1 << 29) + 1, 1 << 30, 0x7FFFFF00};
  for (int left : lefts) {
    if (row_bytes(left, 32, 4) != (left < 32 ? left * 4 : 128)) return 1;
    if (row_bytes(left, 64, 2) != (left < 64 ? left * 2 : 128)) return 2;
    if (left > 0 && left < 128 && row_bytes(-left, 64, 2) > 0) return 3;
  }"""
    run(tmp_path, body)
    # and the kernel counts them this way
    text = open(os.path.join(CSRC, "fp8_block_gemm.cu")).read()
    assert text.count("row_bytes(") == 2 and "cols * 2" not in text
