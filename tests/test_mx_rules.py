"""How calls of hyp_mx.h are cut into workgroups, compiled on the host on its own: every key has a part and every touched block a tile, parts fit
LDS, the number of workgroups stays small; and what the compiler made of the kernels."""
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
                        f"-I{ROOT / 'paper_2511_14450_amd/csrc'}", str(ROOT / "tests/rules/mx_driver.cpp"), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(lines):
        r = subprocess.run([str(exe)], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr[-2000:]
        return [[int(v) for v in line.split()] for line in r.stdout.splitlines()]
    return run


def test_token_parts(ask):
    rng = random.Random(1)
    cases = []
    for _ in range(900):
        features, formats = rng.choice((1, 2, 3, 4, 5, 8)), rng.choice((34, 50, 66))
        cases.append((rng.choice((1, 2, 8, 64, 255, 320, 5000, 1 << 23)), rng.choice((1, 4, 16, 17, 24, 71, 256)), rng.choice((1, 15, 17, 256, 1023, 1024, 9000, 131072, (1 << 30) - 1)),
                      rng.choice((16, 32, 48, 128, 1 << 20)), rng.choice((0, 0, 16, 32, 256)), features * formats, features, rng.choice((0, 1))))
    for (tiles, head_tiles, unit, units, parts), (pairs, group, keys, page, block, _, features, f32) in zip(ask([("token " + " ".join(map(str, c))) for c in cases]), cases):
        assert tiles in (1, 2) and 16 * tiles * head_tiles >= group > 16 * tiles * (head_tiles - 1)
        assert tiles == 1 or (group > 16 and features <= 4 and not f32)    # the kernels there are
        items = pairs * head_tiles
        assert unit == (4 if page % 32 or block == 16 else 5)             # a unit lies in one page and block
        assert 1 <= units <= 256 and units % 8 == 0
        assert units * parts << unit >= keys > units * (parts - 1) << unit  # all keys have a part, and every part has keys
        if keys < 512:
            assert parts == 1
        if parts > 1 and units < 256:                                     # what LDS holds forces more
            assert items * parts <= 512 and keys // parts >= 248          # a part is rounded up to eight units


def test_score_tiles(ask):
    for (turns, tiles), (pairs, blocks) in zip(ask(["scores 1 257", "scores 64 2048", "scores 64 700", "scores 100000 5000"]), ((1, 257), (64, 2048), (64, 700), (100000, 5000))):
        assert turns in (1, 2, 4) and 64 * turns * tiles >= blocks > 64 * turns * (tiles - 1)
        assert turns == 1 or pairs * tiles >= 512


def test_every_block_that_rows_touch_has_a_tile(ask):
    rng = random.Random(2)
    cases = []
    for _ in range(300):
        n, block = rng.choice((1, 2, 5, 40)), rng.choice((16, 64, 256))
        counts = [rng.choice((0, 1, 1, block - 1, block, block + 1, rng.randrange(1000))) for _ in range(n)]
        cases.append((counts, [rng.randrange(5000) for _ in counts], block))
    got = ask([f"write {sum(c)} {len(c)} {b} 0" for c, _, b in cases])
    for (tiles,), (counts, first, block) in zip(got, cases):
        start = [sum(counts[:i]) for i in range(len(counts) + 1)]
        begins = [s // block + 2 * i for i, s in enumerate(start[:-1])] + [tiles]
        for b, (n, j) in enumerate(zip(counts, first)):
            touched = (j + n - 1) // block - j // block + 1 if n else 0
            assert touched <= begins[b + 1] - begins[b], (counts, first, block)
    assert ask(["write 7 7 64 1"]) == [[7]]


def test_kernels_do_not_spill(kernels):  # noqa: F811
    found = {name: k for name, k in kernels.items() if re.search(r"k_mx_", name)}
    assert sum("k_mx_token" in name for name in found) == 64 + 16   # two types, eight sizes, two formats of either; up to 128 bf16 features for two tiles of heads
    for name, k in found.items():
        assert k["scratch"] == 0 and k["spilled"] == 0, (name, k)
        if "k_mx_token" in name and "k_mx_tokenIfLi7" not in name and "k_mx_tokenIfLi8" not in name:
            assert k["vgprs"] <= 256, (name, k)                # two waves a SIMD
