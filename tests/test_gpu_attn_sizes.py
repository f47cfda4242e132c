"""Head sizes, numbers of parts and lengths at which the operators of hyp_attn.h take a code path of their own, and problems drawn at random."""
import math
import random

import pytest
import torch

from tests.test_gpu_attn import BF, F32, NAN, Problem, check_prompt, check_token

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [1, 2, 3, 4, 31, 65, 66, 97, 126, 127, 129, 130, 132, 255])
def test_head_sizes(dtype, d):
    # parts are joined by one, two or four features a lane, or one at a time where none of these fits
    check_token(Problem(d, dtype, 4, 2, d, held=[37, 0, 140, 600], prefix=75))
    check_prompt(Problem(d + 1, dtype, 4, 2, d, held=[700, 40], rows=[2, 3], prefix=300), last=2)
    check_prompt(Problem(d + 2, dtype, 3, 1, d, held=[70, 140], rows=[70, 9], docs=3))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d", [64, 128, 99, 136])
def test_more_parts_than_a_wave_has_lanes(dtype, d):
    # one request of one KV head: 256 keys a part, so some 80 and 120 of them
    check_token(Problem(d, dtype, 2, 1, d, held=[20000], prefix=0))
    check_token(Problem(d + 1, dtype, 2, 1, d, held=[21], prefix=30000))
    check_token(Problem(d + 2, dtype, 1, 1, d, held=[17000], prefix=16500, cap=20.0))


def drawn(seed):
    rng = random.Random(seed)
    nkv = rng.choice((1, 2, 3, 5))
    nq, d = nkv * rng.choice((1, 1, 2, 3, 4, 7, 16, 33)), rng.choice((8, 16, 40, 64, 64, 72, 96, 104, 128, 128, 160, 192, 256, rng.randrange(1, 257)))
    n = rng.choice((1, 1, 2, 3, 5, 9))
    held = [int(math.exp(rng.uniform(0, math.log(600 if n < 5 else 90)))) - 1 for _ in range(n)]
    rows = [min(h + rng.choice((0, 0, 0, 2)), rng.choice((h, h, 0, 1, 17, h // 2))) for h in held]
    rows = [r if d * nq < 2000 else min(r, 60) for r in rows]
    more = dict(prefix=rng.choice((0, 0, 1, 31, 64, 130, 500)), cap=rng.choice((0.0, 0.0, 1.5, 30.0)), slopes=rng.random() < 0.4, pos=rng.random() < 0.4, docs=rng.choice((None, None, 1, 4)),
                page=rng.choice((0, 0, 1, 8, 64, 256, 1024)), layout=rng.choice(("heads", "heads", "tokens", "odd")), sigma=rng.choice((0.3, 1.0, 1.0, 3.0)))
    see = [rng.choice((0, -3, 5, h, 10 ** 6)) for h in held] if rng.random() < 0.4 else None
    return dict(nq=nq, nkv=nkv, d=d, held=held, **more), rows, see, rng.choice((0, 0, 1, 3, 40)), rng.choice((BF, BF, F32))


@pytest.mark.parametrize("seed", range(60))
def test_drawn_problems(seed):
    args, rows, see, last, dtype = drawn(seed)
    check_token(Problem(seed, dtype, **args), totals=seed % 3 != 0)
    check_prompt(Problem(seed + 1, dtype, **args, rows=rows, see_all=see), last=last)
