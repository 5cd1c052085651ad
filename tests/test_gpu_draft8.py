"""The 8-bit draft model as a whole: its step against the plain decoder in 64 bits, windows against single tokens, its draft loop
eagerly and as a graph, and rounds in which a model drafts in 8 bits for itself in bf16."""
import pytest
import torch

import q8_ref
from paper_2411_00853_amd import workload as wl

pytestmark = pytest.mark.gpu

SHAPE = wl.ModelShape(2, 384, 6, 2, 64, 640, 1000)          # widths of three and five blocks, three query heads to a kv head
WIDE = wl.ModelShape(2, 256, 2, 1, 128, 300, 777)            # an FFN and a vocabulary that end inside a block


def round_rows(y):
    q, s = q8_ref.quantise_rows(y)
    y8 = q.double().view(q.shape[0], -1, 128) * s.double().t()[..., None]
    return y8.reshape(q.shape)[:, :y.shape[1]]


def round_weight(w):
    q, s = q8_ref.quantise_weight(w)
    return q.double() * s.double().repeat_interleave(128, 0)[:w.shape[0]].repeat_interleave(128, 1)[:, :w.shape[1]]


def round_pages(x):
    """Keys or values [n][heads][hd] of positions 0 .. n-1, written at once."""
    out = torch.empty_like(x)
    for t in range(0, x.shape[0], 32):
        s = q8_ref.pow2_scale(x[t:t + 32].abs().amax((0, 2)))[:, None]
        out[t:t + 32] = (x[t:t + 32] / s).float().to(q8_ref.F8).double() * s
    return out


def plain_logits(shape, w, tokens, eight_bit):
    """Logits of every position of tokens [n] in fp64, with the roundings to 8 bits (eight_bit) or without any."""
    from paper_2411_00853_amd.draft8 import rope_table
    n, hd, eps = len(tokens), shape.head_dim, shape.rms_eps
    norm = lambda x, g: x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * g.double()
    pages = round_pages if eight_bit else lambda x: x

    def product(x, m):
        x, m = (round_rows(x), round_weight(m)) if eight_bit else (x, m.double())
        return x @ m.t().contiguous()

    cs = rope_table(n, hd, shape.rope_theta, w["tok_embed"].device)
    x = w["tok_embed"].double()[tokens.long()]
    for lw in w["layers"]:
        q, k, v = product(norm(x, lw["attn_norm"]), lw["w_qkv"]).split((shape.d_q, shape.d_kv, shape.d_kv), -1)
        q = q8_ref.rotate(q.reshape(n, -1, hd), cs)
        k = q8_ref.rotate(k.reshape(n, -1, hd), cs)
        o, _ = q8_ref.attend(q, pages(k), pages(v.reshape(n, -1, hd)), list(range(n)), hd ** -0.5)
        x = x + product(o.reshape(n, -1), lw["w_o"])
        g, u = product(norm(x, lw["ffn_norm"]), lw["w_gate_up"]).chunk(2, -1)
        x = x + product(g * torch.sigmoid(g) * u, lw["w_down"])
    return product(norm(x, w["final_norm"]), w["lm_head"])


def rms(x):
    return float(x.double().pow(2).mean().sqrt())


def model(shape, batch, max_kv, window, **filters):
    from paper_2411_00853_amd.draft8 import Draft8
    w = wl.make_weights(shape, 5, "cuda", std=0.05)
    return w, Draft8(shape, w, batch, max_kv, window, **filters)


@pytest.mark.parametrize("shape", (SHAPE, WIDE))
def test_logits_are_those_of_the_plain_decoder(shape):
    """The roundings to 8 bits (2^-4 of a number at most) decide how far the logits are from the unrounded decoder's; the others, to
    bf16 (2^-8 of a number), and sums in fp32 are a sixteenth of them and less.  So the distance is that of the plain decoder
    with the same 8-bit roundings, up to a quarter (several times the sixteenth, for roundings that fall the other way), and the
    two 8-bit decoders are nearer to each other than either is to the unrounded one."""
    n, batch = 70, 3
    w, d = model(shape, batch, 96, n)
    tokens = wl.Rng(6, "cuda").randint(0, (batch, n), shape.vocab)
    got = d.feed(tokens, torch.zeros(batch, dtype=torch.int32, device="cuda")).double().view(batch, n, -1)
    for b in range(batch):
        exact, plain = (plain_logits(shape, w, tokens[b], on) for on in (False, True))
        assert rms(got[b] - exact) < 1.25 * rms(plain - exact)
        assert rms(got[b] - plain) < rms(plain - exact)


def test_a_window_is_its_tokens_one_by_one():
    """The products and norms of a row do not depend on the others.  A page's scale that grows with a later position rounds the older
    ones once more, so that the two caches differ, by less than the 8-bit roundings do from the unrounded decoder."""
    n, batch = 40, 2
    w, d = model(SHAPE, batch, 64, n)
    tokens = wl.Rng(7, "cuda").randint(0, (batch, n), SHAPE.vocab)
    zero = torch.zeros(batch, dtype=torch.int32, device="cuda")
    whole = d.feed(tokens, zero).view(batch, n, -1)[:, -1].clone()
    for t in range(n):
        one = d.feed(tokens[:, t:t + 1].contiguous(), zero + t)
    for b in range(batch):
        exact = plain_logits(SHAPE, w, tokens[b], False)[-1]
        assert rms(one[b] - whole[b]) < rms(whole[b] - exact)


def test_draft_loop_as_a_graph():
    batch, K, n = 3, 4, 33
    _, d = model(SHAPE, batch, 64, n, temperature=0.8, top_k=50, top_p=0.9, min_p=0.01)
    rng = wl.Rng(8, "cuda")
    context = rng.randint(0, (batch, n), SHAPE.vocab)
    kv_len = torch.full((batch,), n - 1, dtype=torch.int32, device="cuda")
    d.feed(context[:, :n - 1].contiguous(), torch.zeros_like(kv_len), logits=False)
    prev, last = context[:, -2].contiguous(), context[:, -1].contiguous()
    u = rng.uniform(1, (3, K, batch))
    eager = []
    for r in range(3):
        tokens = torch.empty((batch, K), dtype=torch.int32, device="cuda")
        logits = torch.empty((batch, K, SHAPE.vocab), device="cuda")
        d.propose(prev, last, kv_len, u[r], tokens, logits)
        eager.append((tokens, logits))
        kept = torch.isfinite(logits)
        assert torch.all(kept.gather(2, tokens.long()[..., None]))
        assert int(kept.sum(-1).max()) <= 50
    tokens, logits = torch.zeros_like(eager[0][0]), torch.zeros_like(eager[0][1])
    uu = u[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        d.propose(prev, last, kv_len, uu, tokens, logits)
    for r in (0, 2, 1, 0):
        uu.copy_(u[r])
        logits.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tokens, eager[r][0]) and torch.equal(logits, eager[r][1])


def test_rounds_of_a_model_that_drafts_for_itself():
    """Acceptance is one less the distance of the two distributions; with logits of root mean square s (0.05 sqrt(384) = 0.98), off by
    about a sixth of it, half the mean of |p - q| is about 0.4 * 0.156 * 0.98 = 0.061.  240 proposals, the mean of accepted ones
    at least 0.939 ** 1..4 of the first to the fourth: 0.86 in the mean, 0.1 below it for their number (over four standard deviations)."""
    from paper_2411_00853_amd.draft8 import Rounds
    batch, K, n, R = 4, 4, 50, 15
    w, d = model(SHAPE, batch, n + (R + 1) * (K + 1), 16)
    rounds = Rounds(SHAPE, w, d, K)
    rng = wl.Rng(9, "cuda")
    rounds.feed(rng.randint(0, (batch, n), SHAPE.vocab))
    assert rounds.kv_len.tolist() == [n - 1] * batch
    kept, length = 0, torch.full((batch,), n - 1)
    for r in range(R):
        rounds.propose(rng.uniform(10 + r, (K, batch)))
        rounds.verify(rng.uniform(100 + r, (batch, K + 1)), 1.0)
        a = rounds.n_accepted.cpu()
        assert torch.all((a >= 0) & (a <= K))
        out = rounds.out.cpu()
        for b in range(batch):
            assert out[b, :a[b]].tolist() == rounds.tokens[b, :a[b]].tolist()
            assert int(rounds.last[b]) == out[b, a[b]] and (a[b] == 0 or int(rounds.prev[b]) == out[b, a[b] - 1])
        length += a + 1
        assert rounds.kv_len.cpu().tolist() == length.tolist()
        kept += int(a.sum())
    from paper_2411_00853_amd import binding as sv
    sv.spec_verify_poll(rounds.handle)
    assert kept / (R * batch * K) > 0.76
