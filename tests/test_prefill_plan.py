"""The kernels and splits that the GPU tests of the prompt's attention reach: the plan is
host code with a header of its own, compiled here.  Its costs can be fitted anew without a
kernel losing its tests unnoticed."""
import os
import shutil
import subprocess

import pytest

import test_gpu_prefill
import test_gpu_prefill_plans

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("needs g++")
    exe = str(tmp_path_factory.mktemp("plan") / "prefill_plan")
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2606_29563_amd", "csrc"),
                           os.path.join(ROOT, "tests", "c", "prefill_plan.cpp"), "-o", exe])

    def of(cases):
        """[(kernel, splits)] of cases (b, H, G, d, q rows, keys, dtype, window, sinks, ...)."""
        lines = []
        for b, H, G, d, nq, nk, dt, window, sinks, *_ in cases:
            window = 0 if window >= nk else window  # as the C interface takes them
            sinks = min(sinks, nk) if window else 0
            lines.append(f"{b} {H} {G} {d} {2 if dt == 'bf16' else 4} {nq} {nk} {window} {sinks}\n")
        got = subprocess.run([exe], input="".join(lines), capture_output=True, text=True, check=True).stdout.split()
        return list(zip(got[::2], map(int, got[1::2])))
    return of


def test_plans_of_the_cases_that_name_them(plan):
    assert plan(test_gpu_prefill_plans.PLANS) == [c[-2:] for c in test_gpu_prefill_plans.PLANS]


def test_every_kernel_and_join_has_a_gpu_test(plan):
    cases = [c[:9] for c in test_gpu_prefill.CASES + test_gpu_prefill.LONG + test_gpu_prefill_plans.PLANS]
    reached = set()
    for (_, _, _, d, _, _, dt, *_), (kernel, splits) in zip(cases, plan(cases)):
        reached.add((kernel, d, splits > 1))
        if splits > 1:
            reached.add(("join", dt, d, min(n for n in (2, 4, 8, 64) if splits <= n)))
    kernels = [(k, d) for k in ("rows16", "rows16_keys", "rows32_half", "rows32_keys", "rows32_keys4") for d in (64, 128)]
    want = {(k, d, split) for k, d in kernels + [("rows32", 128), ("few", 128)] for split in (False, True)}
    want |= {("join", dt, d, n) for dt in ("bf16", "f32") for d in (64, 128) for n in (2, 4, 8, 64)}
    assert want <= reached, want - reached
