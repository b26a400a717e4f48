"""What the products' plans decide, asked of the library's own code by a program that is compiled here for the host."""
import os
import random
import subprocess

import pytest

from paper_1909_07588_b200 import build

PROGRAM = r"""
#include "laq_ops_gradients.cu"
using namespace laq::ops;
// "gradient M N K": together or apart, the widths of the tiles, and the estimate of one launch in hundredths of that of two.  "linear8 M N K", "gated M F K": the form.
int main() {
  char what[16];
  long long M, N, K;
  while (scanf("%15s %lld %lld %lld", what, &M, &N, &K) == 4) {
    if (!strcmp(what, "gradient")) {
      const Plan dx = make_plan(M, K, N, false, true, true, false, false), dw = make_plan(N, K, M, true, true, false, false, false);
      const Form form = both_form(M, N, K);
      printf("%s %d %d %d %d\n", both_pay(M, N, K) ? "together" : "apart", form.nt, dx.nt, dw.nt, (int)(100 * form.cost / (dx.cost + dw.cost + 4000)));
    } else {
      const bool gated = !strcmp(what, "gated");
      const Plan p = make_plan(M, gated ? 2 * N : N, K, false, false, true, false, false, gated ? kGated : kCodes);
      printf("%s %d %d\n", p.pair ? "pair" : p.swap ? "transposed" : "lone", p.nt, p.split);
    }
  }
}
"""


@pytest.fixture(scope="session")
def plans(tmp_path_factory):
    where = tmp_path_factory.mktemp("plans")
    (where / "plans.cu").write_text(PROGRAM)
    flags = [f for f in build.NVCC_FLAGS if f not in ("-shared", "-O3", "-lineinfo")]
    subprocess.run([os.environ.get("NVCC", "nvcc")] + flags + ["-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "-o", str(where / "plans"),
                    str(where / "plans.cu"), "-lcuda"], check=True, capture_output=True)

    def ask(lines):
        out = subprocess.run([str(where / "plans")], input="\n".join(" ".join(map(str, l)) for l in lines) + "\n", capture_output=True, text=True, check=True)
        return [[int(t) if t.isdigit() else t for t in l.split()] for l in out.stdout.splitlines()]
    return ask


def test_two_products_in_one_launch_of_narrower_tiles(plans):
    """Measured with narrower ones: 8192 x 11008 x 784 491 us for 363 apart, 1024 x 11008 x 2048 139 for 122, 8192 x 2048 x 1024 106 for 95."""
    sizes = [(M, N, K) for M in (16, 100, 300, 1024, 4096, 8192) for N in (64, 200, 512, 2048, 8192, 11008) for K in (64, 256, 784, 1024, 2048, 8192)]
    answers = plans([("gradient",) + s for s in sizes])
    assert len(answers) == len(sizes)
    joined = [(s, a) for s, a in zip(sizes, answers) if a[0] == "together"]
    assert len(joined) > 50
    for size, (_, nt, dx, dw, share) in joined:
        assert share < 85 or nt >= dx and nt >= dw, size
    slower = [(8192, 11008, 784), (4096, 11008, 784), (1024, 11008, 2048), (8192, 2048, 1024), (2048, 8192, 1024), (256, 2048, 8192)]
    assert all(a[0] == "apart" for a in plans([("gradient",) + s for s in slower]))
    faster = [(4096, 4096, 512), (8192, 4096, 1024), (8192, 8192, 2048), (300, 512, 1024), (200, 200, 4096), (1817, 176, 1808)]
    assert all(a[0] == "together" for a in plans([("gradient",) + s for s in faster]))


WIDTHS = {"gated": {"pair": (128, 256), "lone": (64, 128, 192, 256), "transposed": (16, 32, 64, 96, 112, 128)},
          "linear8": {"pair": (128, 256), "lone": (64, 128), "transposed": (16, 32, 64, 96, 112, 128)}}


@pytest.mark.parametrize("kind", sorted(WIDTHS))
def test_every_form_is_compared(plans, kind):
    """The sizes of tests/test_gpu_ops_forms.py take the forms that stand there, which are all that the plans give."""
    from tests import test_gpu_ops_forms as forms
    listed = forms.GATED if kind == "gated" else forms.LINEAR8
    assert dict(zip(listed, map(tuple, plans([(kind,) + s for s in listed])))) == listed
    forms_of = {(form, nt) for form, nt, _ in listed.values()}
    assert forms_of == {(form, nt) for form, widths in WIDTHS[kind].items() for nt in widths}
    rng = random.Random(1)
    sizes = [tuple(int(2 ** rng.uniform(a, b)) for a, b in ((2.4, 13), (0, 13.5), (0, 14))) for _ in range(5000)]
    assert {(a[0], a[1]) for a in plans([(kind,) + s for s in sizes])} <= forms_of
    splits = {(form, nt, split > 1) for form, nt, split in listed.values()}
    if kind == "gated":                # whole and split sums end differently
        assert splits >= {("lone", nt, s) for nt in (64, 128, 192, 256) for s in (False, True)} | {("transposed", 128, False), ("transposed", 128, True)}


def test_gradients_that_share_a_launch(plans):
    """The sizes of tests/test_gpu_ops_gradients_forms.py."""
    from tests.test_gpu_ops_gradients_forms import SIZES
    got = plans([("gradient",) + s for s in SIZES])
    assert {s: a[1] if a[0] == "together" else 0 for s, a in zip(SIZES, got)} == SIZES
