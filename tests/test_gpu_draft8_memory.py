"""The 8-bit draft model's loop takes no device memory, and says which windows it takes."""
import pytest
import torch

from paper_2411_00853_amd import workload as wl

pytestmark = pytest.mark.gpu

SHAPE = wl.ModelShape(2, 384, 6, 2, 64, 640, 1000)


def model(batch, window, **filters):
    from paper_2411_00853_amd.draft8 import Draft8
    return Draft8(SHAPE, wl.make_weights(SHAPE, 5, "cuda", std=0.05), batch, 64, window, **filters)


def allocated():
    return torch.cuda.memory_stats()["allocation.all.allocated"]


@pytest.mark.parametrize("filters", [{}, {"top_k": 40, "top_p": 0.9}])
def test_feed_and_propose_allocate_nothing(filters):
    batch, K = 3, 4
    d = model(batch, 8, **filters)
    rng = wl.Rng(8, "cuda")
    context = rng.randint(0, (batch, 9), SHAPE.vocab)
    window, kv_len = context[:, :8].contiguous(), torch.zeros(batch, dtype=torch.int32, device="cuda")
    prev, last = context[:, 7].contiguous(), context[:, 8].contiguous()
    u = rng.uniform(1, (K, batch))
    tokens = torch.empty((batch, K), dtype=torch.int32, device="cuda")
    logits = torch.empty((batch, K, SHAPE.vocab), device="cuda")
    where = kv_len + 8

    def run():
        d.feed(window, kv_len, logits=False)
        d.feed(last.view(batch, 1), where)
        d.propose(prev, last, where, u, tokens, logits)

    run()                       # (the libraries' own first calls)
    torch.cuda.synchronize()
    before = allocated()
    run()
    torch.cuda.synchronize()
    assert allocated() == before


def test_windows_that_do_not_fit():
    d = model(2, 1)
    one = torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    kv_len, u = torch.ones(2, dtype=torch.int32, device="cuda"), torch.zeros((1, 2), device="cuda")
    assert d.feed(one, kv_len).shape == (2, SHAPE.vocab)
    for w in (0, 2):
        with pytest.raises(ValueError, match="window of %d" % w):
            d.feed(torch.zeros((2, w), dtype=torch.int32, device="cuda"), kv_len)
    with pytest.raises(ValueError, match="max_window"):
        d.propose(one[:, 0], one[:, 0], kv_len, u, torch.zeros((2, 1), dtype=torch.int32, device="cuda"), torch.zeros((2, 1, SHAPE.vocab), device="cuda"))
