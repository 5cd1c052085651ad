"""Whole prompts through a model: the operators together, against the plain decoder in 64 bits, and what decodes from the cache they leave."""
import pytest
import torch

import prompt_ref as ref
from paper_2411_00853_amd import binding as sv
from paper_2411_00853_amd import workload as wl
from paper_2411_00853_amd.prompt import Prompt, pack_weights

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16

GROUPED = wl.ModelShape(2, 384, 6, 2, 64, 640, 1000)
WIDE = wl.ModelShape(2, 256, 2, 1, 128, 320, 777)


def plain_logits(shape, w, tokens, rounded):
    """fp64 logits of every position, with the roundings to bf16 that a prompt's pass makes, or without any."""
    n, hd = len(tokens), shape.head_dim
    r = (lambda t: t.to(BF16).double()) if rounded else (lambda t: t)
    norm = lambda x, g: r(x * torch.rsqrt((x * x).mean(-1, keepdim=True) + shape.rms_eps) * g.double())
    x = w["tok_embed"].double()[tokens.long()]
    pos = torch.arange(n, device="cuda")
    for lw in w["layers"]:
        q, k, v = r(ref.product(norm(x, lw["attn_norm"]), lw["w_qkv"])).split((shape.d_q, shape.d_kv, shape.d_kv), -1)
        turn = lambda t: r(ref.rotate(t.reshape(n, -1, hd), pos, shape.rope_theta)).reshape(n, -1)
        o, _, _ = ref.attend(turn(q), turn(k), v, shape.n_kv_heads, hd ** -0.5, [n], [n])
        x = x + ref.product(r(o), lw["w_o"])
        x = x + ref.product(r(ref.product(norm(x, lw["ffn_norm"]), lw["w_gate_up"], act="swiglu")), lw["w_down"])
    return ref.product(norm(x, w["final_norm"]), w["lm_head"])


def rms(x):
    return float(x.double().pow(2).mean().sqrt())


def setup(shape, slots, max_kv, max_rows, pages=0, lookahead=3):
    w = wl.make_weights(shape, 5, "cuda", std=0.05)
    packed = pack_weights(w)
    cfg = sv.make_cfg(shape, slots, max_kv, lookahead)
    nbytes = pages * sv.spec_kv_page_bytes(cfg) if pages else sv.spec_kv_cache_bytes(cfg)
    kv_len = torch.zeros(slots, dtype=torch.int32, device="cuda")
    h = sv.spec_verify_init(cfg, packed, torch.zeros(nbytes, dtype=torch.uint8, device="cuda"), kv_len, paged=bool(pages))
    return w, h, kv_len, Prompt(h, packed, max_rows)


@pytest.mark.parametrize("shape", (GROUPED, WIDE))
@pytest.mark.parametrize("lens", ([70], [5, 130, 1, 33]))
@pytest.mark.parametrize("pages", (0, 30))
def test_logits_and_what_decodes_from_the_cache(shape, lens, pages):
    """Roundings to bf16 decide how far a row's logits are from the unrounded decoder's.  The plain decoder with the same roundings is as far
    from it: its sums are exact ones, so that numbers near the border of two roundings fall the other way, and what follows from those is another
    draw of the same size.  Rows differ in that size by their tokens and lengths, so each is compared with itself.  The error of a
    row is a vector of d_model numbers; with 32 independent directions in it at the least its length scatters by 1 / sqrt(64) =
    0.125, the quotient of two by 0.18, and twice the length is over five times that.  (A term left out shows as some hundred times it.)
    The two share most of their roundings and are nearer to each other than independent ones, sqrt(2) apart, twice that scatter allowed: 1.9.
    Three tokens behind each prompt, scored by the verify step (whose roundings are fewer), are as near."""
    B = len(lens)
    w, h, kv_len, prompt = setup(shape, B + 1, 160, sum(lens) + 3, pages)
    slots = ref.ints([(2 * b + 1) % (B + 1) if B % 2 == 0 else b for b in range(B)])
    tokens = wl.Rng(6, "cuda").randint(0, (sum(lens) + 4 * B,), shape.vocab)
    starts = ref.starts(lens)
    more = tokens[sum(lens):].view(B, 4)
    got = prompt.run(tokens[:sum(lens)], ref.ints(starts), slots, max(lens)).clone()
    for b, s in enumerate(slots.tolist()):
        kv_len[s] = lens[b]
    logits = torch.zeros((4 * B, shape.vocab), device="cuda")
    na, out = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros((B, 4), dtype=torch.int32, device="cuda")
    sv.spec_verify_step(h, [3] * B, torch.full((B, 4), 0.5, device="cuda"), 1.0, na, out, seq_slot=slots, last_token=more[:, 0].contiguous(),
                        draft_tokens=more[:, 1:].contiguous(), draft_logits=torch.zeros((B, 3, shape.vocab), device="cuda"), logits_out=logits)
    sv.spec_verify_poll(h)
    for b, n in enumerate(lens):
        seq = torch.cat((tokens[starts[b]:starts[b + 1]], more[b]))
        exact, plain = (plain_logits(shape, w, seq, on)[n - 1:] for on in (False, True))
        noise = rms(plain[0] - exact[0])
        assert rms(got[b] - exact[0]) < 2 * noise and rms(got[b] - plain[0]) < 1.9 * noise
        assert rms(logits[4 * b:4 * b + 4] - exact[1:]) < 2 * rms(plain[1:] - exact[1:])


def test_prompts_packed_and_one_by_one():
    """Rows do not depend on each other but for the tile shapes their number chooses: the caches are alike up to the roundings."""
    lens = [40, 9, 77]
    _, h, _, prompt = setup(GROUPED, 3, 96, sum(lens))
    tokens = wl.Rng(7, "cuda").randint(0, (sum(lens),), GROUPED.vocab)
    s = ref.starts(lens)
    all_at_once = prompt.run(tokens, ref.ints(s), ref.ints([0, 1, 2]), 77).clone()
    for b, n in enumerate(lens):
        one = prompt.run(tokens[s[b]:s[b + 1]].contiguous(), ref.ints([0, n]), ref.ints([b]))
        assert rms(one[0] - all_at_once[b]) < 0.01 * rms(one[0])


def test_prompt_as_a_graph():
    lens = [40, 9, 51]
    _, h, _, prompt = setup(GROUPED, 3, 128, sum(lens))
    rows = sum(lens)
    tokens, row0, slots = torch.zeros(rows, dtype=torch.int32, device="cuda"), ref.ints(ref.starts(lens)), ref.ints([0, 1, 2])
    prompt.run(tokens, row0, slots)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        prompt.run(tokens, row0, slots)
    for seed, lens in enumerate(([40, 9, 51], [1, 98, 1], [33, 33, 34])):
        fresh = wl.Rng(20 + seed, "cuda").randint(0, (rows,), GROUPED.vocab)
        tokens.copy_(fresh)
        row0.copy_(ref.ints(ref.starts(lens)))
        prompt.logits.zero_()
        graph.replay()
        torch.cuda.synchronize()
        replayed = prompt.logits[:3].clone()
        assert torch.equal(prompt.run(fresh, row0, slots), replayed)
    sv.spec_verify_poll(h)


def test_more_than_there_is_room_for():
    _, h, _, prompt = setup(WIDE, 2, 64, 20)
    with pytest.raises(ValueError, match="at most"):
        prompt.run(torch.zeros(21, dtype=torch.int32, device="cuda"), ref.ints([0, 21]), ref.ints([0]))
    with pytest.raises(ValueError, match="at most"):
        prompt.run(torch.zeros(3, dtype=torch.int32, device="cuda"), ref.ints([0, 1, 2, 3]), ref.ints([0, 1, 0]))


def test_rounds_behind_a_prompt():
    """The 8-bit draft model's rounds accept what they do behind a context that was fed window by window (0.86 of the proposals in the mean,
    0.1 for their number)."""
    from paper_2411_00853_amd.draft8 import Draft8, Rounds
    batch, K, n, R = 4, 4, 50, 15
    w = wl.make_weights(GROUPED, 5, "cuda", std=0.05)
    rounds = Rounds(GROUPED, w, Draft8(GROUPED, w, batch, n + (R + 1) * (K + 1), 16), K, prompt_rows=batch * n)
    rng = wl.Rng(9, "cuda")
    rounds.feed(rng.randint(0, (batch, n), GROUPED.vocab))
    assert rounds.kv_len.tolist() == [n - 1] * batch
    kept = 0
    for r in range(R):
        rounds.propose(rng.uniform(10 + r, (K, batch)))
        rounds.verify(rng.uniform(100 + r, (batch, K + 1)), 1.0)
        assert torch.all(rounds.n_accepted >= 0)
        kept += int(rounds.n_accepted.sum())
    sv.spec_verify_poll(rounds.handle)
    assert kept / (R * batch * K) > 0.76


def bad_calls():
    x, w, y = (torch.zeros(s, dtype=BF16, device="cuda") for s in ((4, 64), (48 * 128,), (4, 48)))
    q, kv = torch.zeros((10, 256), dtype=BF16, device="cuda"), torch.zeros((10, 128), dtype=BF16, device="cuda")
    row0, gain = ref.ints([0, 10]), torch.ones(64, device="cuda")
    gemm = lambda **c: sv.spec_prompt_gemm(**dict(dict(x=x, w_packed=w, y=y), **c))
    attn = lambda **c: sv.spec_prompt_attention(**dict(dict(q=q, k=kv, v=kv, n_q_heads=4, n_kv_heads=2, q_row0=row0, out=torch.empty_like(q), scale=1.0), **c))
    gemm()
    attn()
    h, _, _ = ref.handle(1, 4, 2, 64, 3, 96)
    append = lambda **c: sv.spec_prompt_append(**dict(dict(h=h, layer=0, qkv=torch.zeros((10, 512), dtype=BF16, device="cuda"),
                                                           rotated=torch.zeros((10, 384), dtype=BF16, device="cuda"), row0=row0, seq_slot=ref.ints([0])), **c))
    append()
    V, S = ValueError, sv.SpecError
    return [(V, "x: expected", lambda: gemm(x=x.float())), (V, "x: expected", lambda: gemm(x=torch.zeros((64, 4), dtype=BF16, device="cuda").t())),
            (V, "y: expected 4 rows", lambda: gemm(y=y[:3])), (V, "w_packed", lambda: gemm(w_packed=w[:-1])), (V, "w_packed", lambda: gemm(w_packed=w.half())),
            (V, "bias: expected shape", lambda: gemm(bias=gain)), (V, "bias: expected", lambda: gemm(bias=y[0])),
            (V, "residual: expected shape", lambda: gemm(residual=y[:, :40])), (V, "residual", lambda: gemm(residual=y.half())),
            (V, "activation", lambda: gemm(activation="tanh")), (V, "device tensor", lambda: gemm(x=x.cpu())),
            (S, "multiple of 16", lambda: gemm(activation="swiglu", w_packed=torch.zeros(80 * 128, dtype=BF16, device="cuda"), y=torch.zeros((4, 40), dtype=BF16, device="cuda"))),
            (V, "workspace", lambda: gemm(workspace=x.cpu())),
            (V, "gain: expected shape", lambda: sv.spec_prompt_rmsnorm(x, gain[:5], 1e-5)), (V, "y: expected", lambda: sv.spec_prompt_rmsnorm(x, gain, 1e-5, x.float())),
            (V, "Float or BFloat16", lambda: sv.spec_prompt_rmsnorm(x.half(), gain, 1e-5)),
            (V, "heads", lambda: attn(n_q_heads=3)), (V, "positive", lambda: attn(n_kv_heads=0)), (V, "k: expected", lambda: attn(n_kv_heads=1)),
            (S, "head_dim", lambda: attn(n_q_heads=8, k=q, v=q, n_kv_heads=8)), (V, "v: expected", lambda: attn(v=kv[:9])), (V, "out: expected", lambda: attn(out=q[:9])),
            (V, "k_row0", lambda: attn(k=kv[:9], v=kv[:9])), (V, "k_row0: expected shape", lambda: attn(k_row0=ref.ints([0, 5, 10]))),
            (V, "q_row0", lambda: attn(q_row0=torch.zeros(2, device="cuda"))), (V, "q_row0", lambda: attn(q_row0=ref.ints([]))),
            (V, "rotated", lambda: append(rotated=torch.zeros((10, 256), dtype=BF16, device="cuda"))), (V, "qkv", lambda: append(qkv=q)),
            (V, "seq_slot", lambda: append(seq_slot=ref.ints([0, 1]))), (V, "pos0", lambda: append(pos0=ref.ints([]))),
            (S, "layer", lambda: append(layer=1)), (S, "sequences", lambda: append(row0=ref.ints([0] * 5), seq_slot=ref.ints([0] * 4)))]


@pytest.mark.parametrize("i", range(32))
def test_the_binding_refuses(i):
    calls = bad_calls()
    kind, match, call = calls[i]
    with pytest.raises(kind, match=match):
        call()
    assert len(calls) == 32


def test_tokens_outside_the_vocabulary():
    """They are told by NaN behind them in their prompt; the others do not notice."""
    lens = [20, 9, 31]
    _, h, _, prompt = setup(GROUPED, 3, 96, sum(lens))
    tokens = wl.Rng(7, "cuda").randint(0, (sum(lens),), GROUPED.vocab)
    row0, slots = ref.ints(ref.starts(lens)), ref.ints([0, 1, 2])
    want = prompt.run(tokens, row0, slots).clone()
    for bad in (-1, GROUPED.vocab, 2 ** 31 - 1, -2 ** 31):
        tokens[22] = bad
        got = prompt.run(tokens, row0, slots)
        assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2]) and torch.isnan(got[1]).all()
    with pytest.raises(ValueError, match="tokens: expected int32"):
        prompt.run(tokens.long(), row0, slots)
    with pytest.raises(ValueError, match="tokens: expected int32"):
        prompt.run(tokens[None], row0, slots)


def test_contexts_longer_than_the_prompt_buffers_go_window_by_window():
    from paper_2411_00853_amd.draft8 import Draft8, Rounds
    batch, K, n = 2, 3, 20
    w = wl.make_weights(GROUPED, 5, "cuda", std=0.05)
    rounds = [Rounds(GROUPED, w, Draft8(GROUPED, w, batch, 64, 16), K, prompt_rows=rows) for rows in (0, batch * (n - 1) - 1, batch * (n - 1))]
    context = wl.Rng(9, "cuda").randint(0, (batch, n), GROUPED.vocab)
    for r in rounds:
        r.feed(context)
        assert r.kv_len.tolist() == [n - 1] * batch and torch.equal(r.last, context[:, n - 1]) and torch.equal(r.prev, context[:, n - 2])
        r.propose(torch.full((K, batch), 0.5, device="cuda"))
        r.verify(torch.full((batch, K + 1), 0.5, device="cuda"), 1.0)
        sv.spec_verify_poll(r.handle)
    assert torch.equal(rounds[0].out, rounds[1].out)


def test_the_handle_of_another_device_is_refused():
    h, _, _ = ref.handle(1, 4, 2, 64, 3, 96)
    h.device = 1        # (as if its cache lay there)
    with pytest.raises(ValueError, match="handle"):
        sv.spec_prompt_append(h, 0, torch.zeros((10, 512), dtype=BF16, device="cuda"), torch.zeros((10, 384), dtype=BF16, device="cuda"), ref.ints([0, 10]), ref.ints([0]))


def test_a_closed_handle_is_refused():
    h, _, _ = ref.handle(1, 4, 2, 64, 3, 96)
    h.close()
    with pytest.raises(sv.SpecError, match="NULL handle"):
        sv.spec_prompt_append(h, 0, torch.zeros((10, 512), dtype=BF16, device="cuda"), torch.zeros((10, 384), dtype=BF16, device="cuda"), ref.ints([0, 10]), ref.ints([0]))


def test_rows_behind_the_last_prompt():
    """A padded batch: the rows behind the last prompt, and prompts without rows, change nothing but the tiles that the number of rows chooses."""
    lens = [40, 0, 33]
    rows = sum(lens)
    _, h, _, prompt = setup(GROUPED, 3, 96, rows + 30)
    for buffer in (prompt.x, prompt.h, prompt.qkv, prompt.attn, prompt.act):
        buffer.fill_(float("nan"))
    tokens = wl.Rng(7, "cuda").randint(0, (rows,), GROUPED.vocab)
    padded = torch.cat((tokens, torch.zeros(30, dtype=torch.int32, device="cuda")))
    row0, slots = ref.ints(ref.starts(lens)), ref.ints([0, 1, 2])
    got = prompt.run(padded, row0, slots).clone()
    want = prompt.run(tokens, row0, slots)
    for b in (0, 2):
        assert torch.isfinite(got[b]).all() and rms(got[b] - want[b]) < 0.01 * rms(want[b])
    sv.spec_verify_poll(h)
