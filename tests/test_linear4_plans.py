"""The exact products' cases reach the kernels that they are there for: the library's own rule, built for the host, says which one each is launched with."""
import os
import shutil
import subprocess

import pytest

from test_gpu_linear4_exact import KINDS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host compiler")
    exe = str(tmp_path_factory.mktemp("plan") / "linear4_plan")
    subprocess.run([gxx, "-std=c++17", "-Wall", "-Wextra", "-Werror", os.path.join(ROOT, "tests", "host", "linear4_plan.cpp"), "-o", exe], check=True)
    return lambda cases, units=256: subprocess.run([exe, str(units)] + [str(n) for c in cases for n in c], check=True, capture_output=True,
                                                   text=True).stdout.split("\n")[:-1]


def test_cases_are_launched_as_they_say(plan):
    cases = list(KINDS)
    assert dict(zip(cases, plan(cases))) == KINDS


def test_every_kernel_is_reached_with_groups_of_every_kind():
    kinds = {(kind.rsplit(" ", 1)[0] if kind.startswith("wide") else kind, "128" if group % 128 == 0 else "64" if group == 64 else "other")
             for (_, _, _, group), kind in KINDS.items()}
    for group in ("128", "64", "other"):
        for kind in ["narrow 2", "narrow 8", "narrow 16"] + [f"wide {tiles} {how}" for tiles in (1, 2, 4) for how in ("whole", "shared")]:
            assert (kind, group) in kinds, (kind, group)
    few = {kind: max(-(-ni // group) for (_, ni, _, group), k in KINDS.items() if k == kind) for kind in ("narrow 2", "narrow 8", "narrow 16")}
    assert few["narrow 2"] == few["narrow 8"] == 1024 and few["narrow 16"] > 256    # scales that a workgroup brings in more than one round
    for tiles in (1, 2, 4):                                                          # and in turns along the rows
        assert any(kind.startswith(f"wide {tiles} ") and not kind.endswith(" 1") for kind in KINDS.values())


def test_plans_of_any_sizes_cover_the_rows(plan):
    """One to a million rows and widths up to the largest: the rule answers, and with other numbers of compute units too."""
    sizes = [1, 2, 3, 17, 64, 65, 1000, 4096, 100003, (1 << 19) - 1]
    widths = [1, 31, 32, 255, 257, 4096, 32768, (1 << 24) - 1]
    cases = [(r, ni, no, g) for r in sizes for ni in widths for no in widths for g in (8, 32, 64, 40, 1 << 20)]
    for units in (1, 64, 256, 304):
        got = plan(cases[:1000], units) + plan(cases[1000:2000], units) + plan(cases[2000:], units)
        assert len(got) == len(cases)
        for (r, ni, no, g), kind in zip(cases, got):
            plain = g < 32 or -(-ni // g) > 1024 or ni < 32 or no * -(-ni // g) < 16
            assert (kind == "any") == plain
            assert kind.startswith("narrow") or r > 2 or plain
