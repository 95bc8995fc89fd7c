"""Which kernel attends over pages, and into how many ranges: the cases of the tests on the GPU reach the kernels that they are there for."""
import os
import shutil
import subprocess

import pytest

from tests import test_gpu_pages_prompts as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUS = 256  # of an MI355X


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    exe = str(tmp_path_factory.mktemp("plan") / "pages_plan")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fsanitize=undefined", os.path.join(ROOT, "tests", "host", "pages_plan.cpp"), "-o", exe],
                   check=True, capture_output=True)

    def ask(d, f32, seqs, new, width, heads, group, page, window=0, chosen=0):
        line = " ".join(str(int(x)) for x in (d, f32, seqs, new, width, heads, group, chosen > 0, chosen, page, window, CUS))
        r = subprocess.run([exe], input=line, capture_output=True, text=True, timeout=60)
        assert r.returncode == 0 and r.stderr == "", r.stderr
        prompt, splits, tiles = map(int, r.stdout.split())
        return prompt, splits, tiles

    return ask


@pytest.mark.parametrize("case", P.CASES)
def test_prompts_are_given_to_their_kernel(plan, case):
    d, page, _, heads, group, lens, new, window, ranges = case
    width = max(-(-n // page) for n in lens) + 2
    assert plan(d, False, len(lens), max(new), width, heads, group, page, window)[:2] == (1, ranges)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_the_other_tests_of_that_kernel(plan, d):
    for n in (90, 100, 150):
        for new in (67, 70):
            assert plan(d, False, P.SEQS, new, -(-n // P.PAGE) + 2, P.HEADS, 1, P.PAGE, 40 if n == 150 else 0)[0] == 1
    for n, page in ((200 + 3 * 23, 16), (150 + 3 * 23, 32)):
        assert plan(d, False, 24, 70, -(-n // page) + 2, 8, 1, page)[0] == 1


def test_plans_of_ordinary_calls(plan):
    """One token: ranges that fill the card once, one range where there is little; drafts: 32 rows to a workgroup; fp32 and lists of pages
    stay with the kernel for few rows."""
    assert plan(128, False, 1, 1, 1024, 8, 4, 64) == (0, 32, 1)
    assert plan(128, False, 1, 1, 4, 8, 4, 64) == (0, 1, 1)
    assert plan(128, False, 64, 8, 64, 8, 4, 64) == (0, 1, 2)
    assert plan(128, True, 4, 2048, 128, 8, 4, 64)[0] == 0
    assert plan(128, False, 4, 2048, 128, 8, 4, 64, chosen=8)[0] == 0
    assert plan(128, False, 4, 2048, 128, 8, 4, 64)[0] == 1
