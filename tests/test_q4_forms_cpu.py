"""Host-side check of the tiles of the 4-bit products (no GPU): every tile that the rule can choose is in the matrix that
tests/test_gpu_q4_forms.py runs with every group size, with and without zero points, at its edges."""
import os
import re

import paper_2602_06412_amd
from tests.test_gpu_q4_forms import FORMS, tile

# workgroup: rows, columns, waves along the reduction
SHAPE = {"16x16,1x16": (16, 16, 16), "16x32,1x8": (16, 32, 8), "16x48,1x8": (16, 48, 8), "32x32,1x8": (32, 32, 8), "32x128,4x2": (32, 128, 2)}


def test_the_rule_here_is_the_rule_of_the_source():
    path = os.path.join(os.path.dirname(paper_2602_06412_amd.__file__), "csrc", "gemm_q4.hip")
    text = re.sub(r"\s+", " ", open(path).read().replace("\\", " "))
    rule = re.search(r"do \{ if \(rows16 >= 3.*?\} while \(0\)", text).group(0)
    assert re.findall(r"if \((.*?)\) Q4_RUN", rule) == [
        "rows16 >= 3 && (int64_t)sl_cdiv(n, 128) * sl_cdiv(m_upper, 32) >= 192", "rows16 >= 3",
        "rows16 == 1 && tiles_n <= 256 && blocks_k >= 16", "tiles_n * rows16 <= 512"]
    # (MT, CT, WN, WK of each, in the order of the conditions)
    assert re.findall(r"Q4_RUN\(GS, (\d+), (\d+), (\d+), (\d+), \d+\)", rule) == [
        ("2", "2", "4", "2"), ("2", "2", "1", "8"), ("1", "1", "1", "16"), ("1", "2", "1", "8"), ("1", "3", "1", "8")]


def test_every_reachable_tile_is_in_the_matrix():
    reached = {tile(n, k, m) for n in (1, 688, 4096, 12288, 24576) for k in (8, 256, 688, 4096, 12288) for m in (1, 16, 17, 32, 33, 61, 100, 224, 1000)}
    assert reached == set(FORMS) == set(SHAPE)
    for form, cases in FORMS.items():
        rows, cols, waves = SHAPE[form]
        assert all(tile(n, k, bound) == form and 1 <= m <= bound for n, k, m, bound in cases)
        blocks = [-(-k // 128) for _, k, _, _ in cases]
        assert any(b > waves for b in blocks) and any(b % waves for b in blocks)               # several steps, waves without a block
        assert any(k % 128 for _, k, _, _ in cases)                                            # a block that ends early
        assert any(n % cols and n % 16 for n, _, _, _ in cases)                                # a tile that ends early
        assert any(m % rows for _, _, m, _ in cases) and any(m < bound for _, _, m, bound in cases)
