"""Which calls of attn_received go by pairs of blocks: those that the GPU tests of that form make, and the rule's two sides."""
import pathlib
import shutil
import subprocess

import pytest

from tests import attn_received_cases as cases

ROOT = pathlib.Path(__file__).resolve().parents[1]


@pytest.fixture(scope="module")
def pairs(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no host compiler")
    exe = tmp_path_factory.mktemp("forms") / "driver"
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        f"-I{ROOT / 'paper_2511_14450_amd/csrc'}", str(ROOT / "tests/rules/span_forms_driver.cpp"), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(calls):
        r = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in calls) + "\n", capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr
        return [line == "1" for line in r.stdout.split()]
    return run


def test_the_gpu_tests_of_pairs_of_blocks_take_that_form(pairs):
    calls = [(c["most"], c["last"], c["requests"], c["nkv"], c["nq"] // c["nkv"]) for c in cases.ALL]
    taken = dict(zip(map(cases.name, cases.ALL), pairs(calls)))
    assert all(taken.values()), taken
    # and are of every size that the form is built for, aligned and not, with odd and even numbers of blocks of 64 and of 128 keys
    assert {d for c in cases.ALL for d in (64, 96, 128, 256) if c["d"] == d} == {64, 96, 128, 256} and any(c["d"] % 8 for c in cases.ALL)
    for size in (64, 128):
        assert {(-(-c["most"] // size)) % 2 for c in cases.ALL} == {0, 1}


def test_both_sides_of_the_rule(pairs):
    assert pairs([(2048, 0, 8, 8, 4), (4500, 0, 1, 10, 4), (300, 200, 42, 2, 4), (300, 0, 40, 2, 4)]) == [True] * 4
    # the last rows alone, up to half; few rows; fewer than 160 pairs
    assert pairs([(2048, 512, 8, 8, 4), (300, 150, 42, 2, 4), (300, 0, 80, 2, 1), (3500, 0, 1, 10, 4), (300, 0, 39, 2, 4), (256, 0, 159, 1, 4)]) == [False] * 6
    # sizes at the end of their range do not overflow
    assert pairs([((1 << 30) - 1, 0, (1 << 24) - 1, 1, 256), ((1 << 30) - 1, (1 << 31) - 1, 1, (1 << 24) - 1, 256), (1, 1, 1, 1, 1)]) == [True, True, False]
