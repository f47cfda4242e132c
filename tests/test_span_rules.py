"""How calls of hyp_attn.h are cut into workgroups, compiled on the host on its own: every part has keys, all rows have a tile, the
number of parts stays small, and few workgroups are cut further; and what the compiler made of the kernels."""
import pathlib
import random
import re
import shutil
import subprocess

import pytest

from tests.test_code_objects import kernels, objects  # noqa: F401

ROOT = pathlib.Path(__file__).resolve().parents[1]


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no host compiler")
    exe = tmp_path_factory.mktemp("rules") / "driver"
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-Werror", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        f"-I{ROOT / 'paper_2511_14450_amd/csrc'}", str(ROOT / "tests/rules/span_driver.cpp"), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(lines):
        r = subprocess.run([str(exe)], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr[-2000:]
        return [[int(v) for v in line.split()] for line in r.stdout.splitlines()]
    return run


def test_prompt_parts(ask):
    rng = random.Random(1)
    cases = [(rng.choice((1, 2, 3, 40, 255, 256, 5000)), rng.choice((1, 2, 7, 8, 9, 64, 4000, 1 << 25)), rng.choice((2, 4))) for _ in range(300)]
    for (splits,), (groups, stages, fewest) in zip(ask([f"prompt {g} {s} {f}" for g, s, f in cases]), cases):
        assert 1 <= splits <= 64
        assert splits == 1 or stages // splits >= fewest       # no part is shorter
        assert splits == 1 or groups * splits <= 512
        if groups < 256 and stages >= 128 * fewest:            # long keys fill the chip
            assert groups * splits > 256 or splits == 64


def test_token_parts(ask):
    rng = random.Random(2)
    cases = [(rng.choice((1, 2, 9, 33, 500)), rng.choice((1, 2, 8, 10)), rng.choice((1, 4, 5, 32, 33, 256)), rng.choice((1, 31, 257, 5000, (1 << 30) - 1)),
              rng.choice((0, 1, 129, 8192, (1 << 30) - 1)), rng.choice((2, 4)), rng.choice((32, 64))) for _ in range(400)]
    for (wide, pre_tiles, pre_splits, tiles, splits), (n, heads, group, most, prefix, waves, stage) in zip(
            ask([("token " + " ".join(map(str, c))) for c in cases]), cases):
        assert tiles * 32 >= group > (tiles - 1) * 32
        assert 1 <= splits <= -(-most // (32 * waves))          # every part has a stage
        # parts are an even share of all keys for 512 workgroups, or 256 keys: each side is rounded up once an item
        assert splits * n * heads * tiles + pre_splits * pre_tiles * heads <= 512 + n * heads * tiles + pre_tiles * heads
        if prefix == 0:
            assert pre_tiles == pre_splits == 0
            continue
        tile = 32 * waves if wide else 32
        assert pre_tiles * tile >= n * group > (pre_tiles - 1) * tile
        assert 1 <= pre_splits <= -(-prefix // (stage if wide else 32 * waves))


def test_kernels_keep_their_waves_and_do_not_spill(kernels):  # noqa: F811
    # bf16 rows of up to 128 features and f32 ones of up to 96 in 16-byte pieces keep two waves a SIMD
    def pick(pattern):
        got = {name: k for name, k in kernels.items() if re.search(pattern, name)}
        assert got, pattern
        return got
    for name, k in pick(r"k_span_(prompt|token|received|join)I|k_evict_").items():
        assert k["scratch"] == 0, (name, k)
    for name, k in pick(r"k_span_(prompt|token)It?f?Li[468]ELb1E").items():
        assert k["vgprs"] <= 256 and k["spilled"] == 0, (name, k)
