"""The serving example: the order of its streams on the host, and that it runs."""
import contextlib

import pytest
import torch

from paper_2506_17615_amd import serving


class _Streams:
    """In place of torch.cuda: which stream has been given what, and what each waits for."""

    def __init__(self):
        self.made, self.now = 0, 0
        self.seen = {0: {"before"}}             # per stream: what is done before anything given to it from here on
        outer = self

        class Stream:
            def __init__(self, number=None):
                if number is None:
                    outer.made += 1
                    number = outer.made
                    outer.seen[number] = set()
                self.number = number

            def wait_stream(self, other):
                outer.seen[self.number] |= outer.seen[other.number]

        class CUDAGraph:
            pass

        self.Stream, self.CUDAGraph = Stream, CUDAGraph
        self.steps = []

    def current_stream(self):
        return self.Stream(self.now)

    @contextlib.contextmanager
    def stream(self, stream):
        last, self.now = self.now, stream.number
        yield
        self.now = last

    @contextlib.contextmanager
    def graph(self, graph):
        self.steps.append("capture")
        yield

    def step(self):
        self.steps.append(set(self.seen[self.now]))
        self.seen[self.now].add("step")


def test_the_first_step_waits_for_what_the_current_stream_was_given(monkeypatch):
    fake = _Streams()
    monkeypatch.setattr(serving.torch, "cuda", fake)
    serving.captured(fake.step)
    first, capture, _ = fake.steps
    assert "before" in first, "the tensors that the step reads were made on the current stream"
    assert capture == "capture" and "step" in fake.seen[0], "the current stream goes on after the step"


@pytest.mark.gpu
def test_the_example_runs(capsys):
    serving.main()
    lines = capsys.readouterr().out.splitlines()
    assert len(lines) == 2 and lines[0].startswith("prompts of [700, 1500, 64, 1] tokens") and lines[1].startswith("decode of 4 sequences")


@pytest.mark.gpu
def test_a_captured_step_reads_what_was_made_just_before():
    rows = torch.arange(1 << 20, device="cuda")
    table, out = torch.randn(1 << 20, device="cuda"), torch.zeros(1 << 20, device="cuda")
    graph = serving.captured(lambda: out.copy_(table[rows]))
    assert torch.equal(out, table)
    for _ in range(3):
        table.normal_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, table)
