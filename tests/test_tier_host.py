"""A tier's nodes with tasks that stay queued until they are told to end: where equal nodes' work goes does not depend on how fast the device or the
host is.  No GPU: the stage's two calls, streams and events are stand-ins, the bookkeeping and the choice are the tier's and the library's."""
import contextlib

import pytest
import torch

from oracle import hyperion_plan as op
from paper_2511_14450_amd import binding
from paper_2511_14450_amd.tier import Tier


class Stream:
    def wait_stream(self, other):
        pass


class Event:
    made = []

    def __init__(self):
        self.over = False
        Event.made.append(self)

    def record(self, stream):
        pass

    def query(self):
        return self.over


class Hidden:
    def record_stream(self, stream):
        pass


@pytest.fixture
def tier(monkeypatch):
    monkeypatch.setattr(torch.cuda, "stream", lambda s: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "current_stream", Stream)
    monkeypatch.setattr(torch.cuda, "Event", Event)
    monkeypatch.setattr(binding, "stage_prefill", lambda stage, hidden, lens: torch.full((sum(lens), 4), float(stage)))
    monkeypatch.setattr(binding, "stage_decode_step", lambda stage, h, out: out.copy_(h + 1))
    t = Tier.__new__(Tier)
    t.capacity, t.memory, t.available = [1.0] * 3, [float("inf")] * 3, [True] * 3
    t.streams, t.stages = [Stream() for _ in range(3)], [0, 100, 200]
    t.queues, t.rows, t.decisions = [[] for _ in range(3)], [{} for _ in range(3)], []
    Event.made = []
    return t


def follows_the_oracle(tier):
    for d in tier.decisions:
        assert d["k"] == op.hypsched_rt(d["F_new"], d["m_act"], d["C"], d["M_avail"], d["available"], d["F_run_rem"], d["F_wait"])


def test_queued_work_spreads_over_equal_nodes(tier):
    tasks = [tier.submit(Hidden(), [3], 2, work=1000.0) for _ in range(9)]
    assert [t.node for t in tasks] == [0, 1, 2] * 3
    assert [float(t.out[0, 0]) for t in tasks] == [2.0, 102.0, 202.0] * 3  # each node's own stage
    follows_the_oracle(tier)


def test_a_task_that_is_done_leaves_its_node_free(tier):
    for _ in range(4):  # every task ends before the next one comes: the first of the equal nodes has them all
        assert tier.submit(Hidden(), [3], 2, work=1000.0).node == 0
        Event.made[-1].over = True
    first, second = tier.submit(Hidden(), [3], 2, work=1000.0), tier.submit(Hidden(), [3], 2, work=1000.0)
    assert (first.node, second.node) == (0, 1)
    first.done.over = True
    assert tier.submit(Hidden(), [3], 2, work=1000.0).node == 0
    follows_the_oracle(tier)
