"""Which form a product in four bits takes, and each form against the reference.  The choice is host arithmetic on the sizes (csrc/fp4_form.h), compiled here by
itself: a shape whose form a change of the costs moves, or a form that no shape below takes any more, shows on the host."""
import os
import random
import subprocess

import numpy as np
import pytest

from test_fp4 import _linear, _matrix

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SMS = 148

# few rows: groups of 128 tokens in a tile, CTAs that share K, rings on an SM, tiles of tokens (one or more), stages beyond the ring or not
FORMS = [((1, 128, 256, 16), "few 1 1 2 one once"), ((90, 1147, 800, 32), "few 1 1 2 one wrap"), ((357, 101, 96, 16), "few 1 1 2 more once"),
         ((281, 21, 960, 32), "few 1 1 2 more wrap"), ((2, 8355, 1824, 32), "few 1 2 2 one once"), ((2, 5709, 7488, 16), "few 1 2 2 one wrap"),
         ((1041, 685, 2336, 32), "few 1 2 2 more wrap"), ((10, 70, 1920, 32), "few 1 4 2 one once"), ((3, 458, 5888, 32), "few 1 4 2 one wrap"),
         ((1186, 25, 1824, 32), "few 1 4 2 more once"), ((1079, 341, 4480, 16), "few 1 4 2 more wrap"), ((1188, 35, 3968, 32), "few 1 4 2 more wrap"),
         ((129, 130, 320, 16), "few 2 1 1 one once"), ((136, 98, 288, 32), "few 2 1 1 one once"), ((162, 4121, 1632, 32), "few 2 1 1 one wrap"),
         ((11987, 260, 5632, 16), "few 2 1 1 more wrap"), ((207, 8118, 6336, 32), "few 2 2 1 one wrap"), ((134, 75, 2368, 32), "few 2 4 1 one once"),
         ((134, 156, 3520, 16), "few 2 4 1 one once"), ((241, 48, 12768, 16), "few 2 4 1 one wrap"), ((6089, 51, 14336, 16), "few 2 4 1 more wrap"),
         ((128, 256, 512, 16), "pair"), ((250, 400, 1024, 32), "pair"), ((2304, 2560, 256, 32), "pair"), ((3500, 5130, 1248, 16), "pair")]
# (weights too wide to be compared in numpy)
WIDE = [((12, 19445, 12544, 16), "few 1 2 1 one wrap"), ((134, 9066, 2336, 16), "few 2 2 1 one once")]
# 16-bit results by kinds of row boundaries: on 16 bytes, on words, on elements
ROWS = [(2304, 2560), (2304, 2562), (2304, 2561)]

HARNESS = """
#include "fp4_form.h"

#include <cstdio>

int main() {
  int rows, outs, width, block, vec, sms;
  while (std::scanf("%d %d %d %d %d %d", &rows, &outs, &width, &block, &vec, &sms) == 6) {
    const ssdi8::Fp4Form f = ssdi8::fp4_form(rows, outs, width, block, vec != 0, sms);
    const int kblocks = (width + 255) / 256;
    const uint32_t image = (uint32_t)f.n * 512u, least = ssdi8::Fp4Few::stage(f.n, block) * (uint32_t)f.stages;
    // what the kernel relies on: a stage for every CTA, stages and the accumulator's image inside the ring
    if (!f.pair && (f.n % 16 || f.n < 16 || f.n > 256 || f.stages < 1 || f.split > kblocks || image > f.ring || least > f.ring)) return 1;
    if (f.pair) std::printf("pair\\n");
    else
      std::printf("few %d %d %d %s %s\\n", f.n <= 128 ? 1 : 2, f.split, f.ring == ssdi8::Fp4Few::kSmall ? 2 : 1, rows > f.n ? "more" : "one",
                  (kblocks + f.split - 1) / f.split > f.stages ? "wrap" : "once");
  }
}
"""


@pytest.fixture(scope="module")
def form_of(tmp_path_factory):
    d = tmp_path_factory.mktemp("forms")
    (d / "forms.cpp").write_text(HARNESS)
    exe = str(d / "forms")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2608_21952_b200", "csrc"), "-o", exe, str(d / "forms.cpp")], check=True)

    def forms(shapes):
        text = "".join("%d %d %d %d %d %d\n" % (*s, SMS) for s in shapes)
        return subprocess.run([exe], input=text, check=True, capture_output=True, text=True).stdout.split("\n")[:-1]
    return forms


def test_form_of_each_shape(form_of):
    for size in (2, 4):
        got = form_of([(*s, s[1] * size % 16 == 0) for s, _ in FORMS + WIDE])
        assert got == [f for _, f in FORMS + WIDE]
        assert set(form_of([(T, O, 256, 32, O * size % 16 == 0) for T, O in ROWS])) == {"pair"}


def test_every_form_has_a_shape(form_of):
    """sizes over the whole range: no form that the shapes above do not take"""
    r = random.Random(0)
    size = lambda lo, hi: int(round(np.exp(r.uniform(np.log(lo), np.log(hi)))))  # noqa: E731
    shapes = [(size(1, 20000), size(1, 20000), 32 * size(1, 512), r.choice((16, 32)), r.choice((0, 1))) for _ in range(60000)]
    got = set(form_of(shapes))
    assert got <= {f for _, f in FORMS + WIDE}
    # no more than what a draw of 60000 may miss is there without being met
    assert len(got) >= 18


def test_ends_of_the_range(form_of):
    """the largest and the smallest sizes have a form that the kernel can take"""
    most = 0x7fffff00
    for shape in ((1, 1, 32), (most, 1, 32), (1, most, 32), (1, 1, 131072), (256, 1, 131072), (257, 128, 131072), (most, 128, 32), (16, most, 4096)):
        for block in (16, 32):
            assert len(form_of([(*shape, block, 0), (*shape, block, 1)])) == 2


@pytest.mark.gpu
@pytest.mark.parametrize("T,O,K,block", [s for s, _ in FORMS])
def test_form(T, O, K, block):
    _linear(T, O, K, block, "float32", bias=True, seed=T + O)
    if T * O * K < 1 << 30:
        _linear(T, O, K, block, "bfloat16", bias=True, act=1, residual=True, seed=T + O + 1)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float16", "bfloat16", "float32"])
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("T,O", ROWS)
def test_pairs_by_rows(T, O, block, dtype):
    _linear(T, O, 256, block, dtype, bias=True, residual=True, seed=T + O)
    _linear(T, O, 160, block, dtype, act=2, seed=T + O)


@pytest.mark.gpu
@pytest.mark.parametrize("T,O,K,block", [s for s, _ in WIDE])
def test_form_of_wide_weights(T, O, K, block):
    """against products in binary64 of the values on the device"""
    import torch
    from paper_2608_21952_b200 import binding as bd
    x, w = _matrix(T, K, block, 1)[0], _matrix(O, K, block, 2)[0]
    vx, vw = torch.empty(T, K, device="cuda"), torch.empty(O, K, device="cuda")
    bd.ssdi8_fp4_dequantize(x, vx)
    bd.ssdi8_fp4_dequantize(w, vw)
    res, out = torch.randn(T, O, device="cuda"), torch.empty(T, O, device="cuda")
    bd.ssdi8_fp4_linear(x, w, out, residual=res)
    vx, vw = vx.double(), vw.double()
    s, size = vx @ vw.T, vx.abs() @ vw.abs().T
    want = s + res.double()
    # the values' roundings (their step sizes) and those of the product: K of its sum, two of the step sizes, the addition's
    tol = 2.0 ** -24 * ((K + 4) * size + s.abs() + 2 * want.abs())
    assert bool(((out.double() - want).abs() <= tol).all())
