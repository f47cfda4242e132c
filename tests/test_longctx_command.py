"""The command of paper_2511_14450_amd.longctx: which options go together, and runs of the shortest kind."""
import json

import pytest
import torch

from paper_2511_14450_amd import longctx


def options(*argv):
    return longctx._arguments(["one", "phi3_medium"], list(map(str, argv)))


@pytest.mark.parametrize("page_keys", [0, 16, 32, 64, 512])
@pytest.mark.parametrize("read_blocks", [0, 1, 2, 3, 4, 5, 6, 64])
def test_any_number_of_blocks_to_read_goes_with_any_page(read_blocks, page_keys):
    a = options("--read-blocks", read_blocks, "--page-keys", page_keys)
    assert a.block_keys == (min(64, page_keys) if page_keys else 64)
    assert a.sink >= 0 and a.recent >= 0 and a.sink + a.recent <= read_blocks
    assert read_blocks < 5 or (a.sink, a.recent) == (1, 4)
    assert read_blocks == 0 or a.recent >= 1


def test_options_that_are_given_are_taken():
    a = options("--read-blocks", 9, "--sink", 0, "--recent", 2, "--block-keys", 16, "--page-keys", 128)
    assert (a.sink, a.recent, a.block_keys) == (0, 2, 16)
    assert options("--read-blocks", 5, "--recent", 4).sink == 1 and options("--read-blocks", 5, "--recent", 5).sink == 0 and options("--read-blocks", 3, "--sink", 3).recent == 0


@pytest.mark.parametrize("argv", [("--read-blocks", -1), ("--read-blocks", 3, "--sink", 4), ("--read-blocks", 3, "--sink", 2, "--recent", 2), ("--sink", -1), ("--recent", -2),
                                  ("--block-keys", 8), ("--block-keys", 48), ("--block-keys", 8192), ("--block-keys", 64, "--page-keys", 32), ("--page-keys", 24),
                                  ("--page-keys", 8), ("--requests", 0), ("--prompt", 0), ("--chunk", 0), ("--generate", -1), ("--blocks", 0), ("--k-format", "int8")])
def test_options_that_do_not_go_together_are_refused_by_name(argv, capsys):
    with pytest.raises(SystemExit) as stop:
        options(*argv)
    assert stop.value.code == 2 and "error:" in capsys.readouterr().err


@pytest.mark.gpu
@pytest.mark.parametrize("more", [("--generate", "0"), ("--generate", "1", "--read-blocks", "2", "--page-keys", "16"), ("--generate", "3", "--read-blocks", "1", "--k-format", "e2m1")])
def test_short_runs(more, monkeypatch, capsys):
    monkeypatch.setattr("sys.argv", ["longctx", "--blocks", "1", "--requests", "2", "--prompt", "90", "--chunk", "64", *more])
    longctx.main()
    out = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert out["prompt"] == 90 and out["prompt_ms"] > 0 and 0 < out["cache_mib"] < out["cache_mib_bf16"]
    torch.cuda.empty_cache()
