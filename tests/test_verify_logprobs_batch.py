"""The outputs of the verify forward's log probabilities have the rows of the run that the library is in, whichever call began it."""
import contextlib
import types

import numpy as np
import pytest


class Stream:
    def wait_stream(self, other):
        pass


class Library:
    """A context's run as the library keeps it: a call that it refuses changes nothing, one that fails later has begun its run."""

    def __init__(self):
        self.batch, self.fail, self.shapes = 1, 0, None

    def begin(self, batch):
        if self.fail == -1:
            return -1
        self.batch = batch
        return self.fail

    def pacer_batch(self, h):
        return self.batch

    def pacer_prefill(self, h, p, batch, *a):
        return self.begin(batch)

    def pacer_generate(self, h, p, batch, *a):
        return self.begin(batch)

    def pacer_generate_sched(self, h, p, batch, *a):
        return self.begin(batch)

    def pacer_generate_ar(self, h, p, batch, *a):
        return self.begin(batch)

    def pacer_verify_logprobs(self, h, top, *outputs):
        return 0

    def pacer_strerror(self, rc):
        return b"failed"

    def pacer_last_error(self, h):
        return b""


@pytest.fixture
def ctx(monkeypatch):
    from paper_2602_01274_b200 import build
    build.build_lib()
    import torch
    from paper_2602_01274_b200 import binding
    c = binding.Context.__new__(binding.Context)
    c.cfg, c.device, c.stream, c._h = types.SimpleNamespace(gamma_cap=4), torch.device("cpu"), Stream(), None
    monkeypatch.setattr(binding, "_lib", Library())
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: Stream())
    return c


def shapes(ctx):
    return [tuple(t.shape) for t in ctx.pacer_verify_logprobs(2)]


def rows(n):
    return [(n, 5), (n, 5), (n, 5, 2), (n, 5, 2)]


def test_the_rows_are_those_of_the_current_run(ctx):
    from paper_2602_01274_b200 import binding
    prompt = lambda n: np.ones((n, 3), np.int32)
    ctx.pacer_prefill(prompt(2), 8, 4, 0.5)
    assert shapes(ctx) == rows(2)
    ctx.pacer_generate(prompt(5), 8, 4, 0.5)
    assert shapes(ctx) == rows(5)
    ctx.pacer_generate_sched(prompt(3), 8, np.ones((3, 2), np.int32))
    assert shapes(ctx) == rows(3)
    ctx.pacer_generate_ar(prompt(4), 8)
    assert shapes(ctx) == rows(4)
    for rc, left in ((-1, 4), (-5, 6)):                     # refused: the run before it stays; failed on its way: its run is the current one
        binding._lib.fail = rc
        with pytest.raises(binding.PacerError):
            ctx.pacer_generate(prompt(6), 8, 4, 0.5)
        assert shapes(ctx) == rows(left)


def test_without_a_context():
    from paper_2602_01274_b200 import build
    build.build_lib()
    from paper_2602_01274_b200 import binding
    assert binding._lib.pacer_batch(None) == 0


@pytest.mark.gpu
def test_verify_after_a_run_of_another_batch():
    import torch
    from paper_2602_01274_b200 import binding as b, synth
    cfg = synth.CONFIGS["tiny"]
    pair = synth.make_pair(cfg, seed=0, device="cuda:0")
    ctx = b.Context(b.make_cfg(cfg.target, cfg.draft, 3, 64 + 32 + cfg.gamma_cap + 2, cfg.gamma_cap, cfg.block_b, cfg.rho, 0, cfg.succ_bias))
    b.load_pair(ctx, pair)
    prompts = synth.make_prompts(cfg.target.vocab, 3, 32, seed=3).numpy()
    ctx.pacer_prefill(prompts[:1], 8, cfg.gamma_cap, 0.5)
    ctx.pacer_generate(prompts, 8, cfg.gamma_cap, 0.5)
    assert b._lib.pacer_batch(ctx._h) == 3
    ctx.pacer_verify()
    logp, ent, ids, tlp = ctx.pacer_verify_logprobs(top=4)
    ctx.stream.synchronize()
    assert logp.shape == ent.shape == (3, cfg.gamma_cap + 1) and ids.shape == tlp.shape == (3, cfg.gamma_cap + 1, 4)
    assert torch.isnan(logp).all() and (ids == -1).all()    # (all three sequences have finished: nothing is written)
    with pytest.raises(b.PacerError):
        ctx.pacer_prefill(prompts[:2], 10 ** 6, cfg.gamma_cap, 0.5)
    assert b._lib.pacer_batch(ctx._h) == 3
    ctx.pacer_prefill(prompts[:2], 8, cfg.gamma_cap, 0.5)
    assert b._lib.pacer_batch(ctx._h) == 2
    ctx.close()
