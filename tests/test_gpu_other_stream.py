"""Calls on a stream that is not the current one: their outputs take no memory that queued work still reads, and are not taken while they are read."""
import pytest
import torch

import helpers
import paper_2502_01662_b200 as pkg
from paper_2502_01662_b200 import synth

pytestmark = pytest.mark.gpu

ROWS, V = 6, 200_000
WAIT = 100_000_000      # clocks: some 50 ms


def calls():
    g = torch.Generator("cuda").manual_seed(2)
    x = torch.randn((ROWS, V), generator=g, device="cuda").bfloat16()
    u = torch.rand(ROWS, generator=g, device="cuda")
    top = pkg.top_logits(x, 700)
    w = synth.CONFIGS["cfg1"].scaled(batch=2, vocab=4096, gamma=3)
    inputs = synth.make_inputs(w, "cuda")
    v = helpers.make_verifier(w)
    run = lambda **kw: v.run(inputs["logits"], inputs["drafts"], inputs["proposer"], inputs["seed"], 0, dump_r=True, **kw)  # noqa: E731
    return v, [lambda **kw: pkg.sample(x, u, 0.9, 20, filtered=True, **kw), lambda **kw: pkg.top_logits(x, 700, **kw),
               lambda **kw: pkg.distill_step(x, top["ids"], top["values"], u, top["lse"], **kw), run]


def sizes(out):
    return sorted({t.untyped_storage().nbytes() for t in out.values()})


def same(a, b):
    return all(torch.equal(torch.nan_to_num(a[n].float(), nan=-7.0), torch.nan_to_num(b[n].float(), nan=-7.0)) for n in a)


@pytest.mark.parametrize("which", range(4))
def test_memory_that_queued_work_still_reads(which):
    v, of = calls()
    side = torch.cuda.Stream()
    call = of[which]
    want = call()
    old = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in sizes(want) for _ in range(4)]
    torch.cuda.synchronize()
    torch.cuda._sleep(WAIT)
    kept = [t.clone() for t in old]
    where = {t.data_ptr() for t in old}
    del old
    got = call(stream=side)
    assert not where & {t.untyped_storage().data_ptr() for t in got.values()}
    torch.cuda.synchronize()
    assert all(bool((t == 7).all()) for t in kept) and same(got, want)
    v.close()


@pytest.mark.parametrize("which", range(4))
def test_outputs_that_are_still_read_here(which):
    v, of = calls()
    side = torch.cuda.Stream()
    call = of[which]
    want = call()
    torch.cuda.synchronize()
    got = call(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(WAIT)
    kept = {n: t.clone() for n, t in got.items()}
    del got
    with torch.cuda.stream(side):
        others = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in sizes(want) for _ in range(4)]
    torch.cuda.synchronize()
    assert same(kept, want) and all(bool((t == 7).all()) for t in others)
    v.close()
