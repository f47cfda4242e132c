"""mx_token's cut of a request's keys: how short a part may be, how many workgroups have room at once, and which calls go by two tiles of heads."""
import random

from tests.test_mx_rules import ask  # noqa: F401


def plan(ask, pairs, group, keys, *, page=1 << 20, block=0, features=4, key_bytes=66, f32=False):  # noqa: F811
    (tiles, head_tiles, unit, units, parts), = ask([f"token {pairs} {group} {keys} {page} {block} {features * key_bytes} {features} {int(f32)}"])
    return dict(tiles=tiles, workgroups=pairs * head_tiles * parts, keys=units << unit, parts=parts, last=keys - (parts - 1) * (units << unit), units=units)


def test_parts_are_equal_but_for_the_last_one_of_a_request(ask):  # noqa: F811
    rng = random.Random(4)
    for _ in range(120):
        keys = int(2 ** rng.uniform(0, 21))
        p = plan(ask, rng.choice((1, 4, 24, 200)), rng.choice((1, 8, 24)), keys, page=rng.choice((16, 128)), features=rng.choice((1, 2, 4, 6, 8)), key_bytes=rng.choice((34, 66)), f32=rng.random() < 0.5)
        assert 1 <= p["last"] <= p["keys"] and (p["parts"] == 1 or p["keys"] >= 256)


def test_a_cut_that_leaves_a_part_of_nearly_nothing_is_estimated_as_it_is(ask):  # noqa: F811
    # four parts of 1025 keys would be three, of 512, 512 and 1: two of 768 and 257, or one, by what the longest takes
    assert plan(ask, 1, 4, 1025)["last"] != 1


def test_float_rows_of_wide_heads_have_room_for_one_workgroup_a_cu(ask):  # noqa: F811
    for features in range(1, 9):
        for key_bytes in (34, 50, 66):
            for keys in (1200, 9000, 32768):
                p = plan(ask, 32, 2, keys, features=features, key_bytes=key_bytes, f32=True)
                assert p["workgroups"] <= (512 if features <= 6 else 256) or p["units"] == 256
    # 8 x 32768 keys of four heads: 129 us in 256 workgroups, 92 in 512; 105 and 112
    assert plan(ask, 32, 2, 32768, features=6, f32=True)["workgroups"] == 512
    assert plan(ask, 32, 2, 32768, features=8, key_bytes=34, f32=True)["workgroups"] == 256


def test_of_two_cuts_that_take_as_long_the_one_of_fewer_parts_is_taken(ask):  # noqa: F811
    # bytes bound either: 24 heads of one request of 131072 keys in 128 parts or 256
    assert plan(ask, 1, 24, 131072, page=128)["workgroups"] == 256 and plan(ask, 64, 4, 32768, page=128)["workgroups"] == 256


def test_groups_of_heads_go_by_two_tiles_where_they_were_faster_by_it(ask):  # noqa: F811
    tiles = lambda requests, keys, kv=1, group=24, **more: plan(ask, requests * kv, group, keys, **more)["tiles"]  # noqa: E731
    assert [tiles(*x) for x in ((8, 131072), (8, 65536), (64, 8192), (64, 16384), (8, 131072, 4, 34))] == [2] * 5
    assert [tiles(*x) for x in ((1, 131072), (1, 524288), (2, 262144), (8, 16384), (8, 32768), (32, 4096), (8, 2000))] == [1] * 7
    assert tiles(64, 65536, f32=True) == tiles(64, 65536, features=5) == tiles(64, 65536, group=16) == 1
