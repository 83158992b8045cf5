"""Generation as a user runs it: prefill of a pruned prompt, then decode steps on
the paged cache.

Layer 0's keys and values do not depend on attention: the integer linears are
exact, so the rows that single-token steps append have to be bit for bit those of
one prefill of the whole sequence, whatever kernels the two sizes take. Layer 0's
attention outputs then differ by the two kernels' errors: the prompt's attention
5.2e-4 (vmax + |o|) + 1e-5 (weights and output rounded to fp16), the paged one
2^-11 |o| + 1e-4 vmax. (What follows passes through 4-bit codes, which a difference
of one rounding may move by a step, and is not compared.)"""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gen(p4q):
    from paper_2609_34867_gb300 import generate
    return generate


def _run(gen, graph, new=12, **params):
    c = gen.Config(d=512, heads=4, kv_heads=2, ffn=1024, layers=2, vocab=1000, page=8)
    decoder = gen.Decoder(c, 3)
    rows, rot_pos, end = gen.pruned_prompt(3, c, 5, N=96, K=24, T=5)
    u = torch.rand((new, 3), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    tokens, _, cache = gen.generate(decoder, rows, rot_pos, end, new, u, graph=graph, **params)
    return c, decoder, rows, rot_pos, end, tokens, cache


def test_steps_and_their_graph_give_the_same_tokens(p4q, gen):
    p = torch.full((3,), 0.9, device="cuda")
    a = _run(gen, False, top_p=p)
    b = _run(gen, True, top_p=p)
    assert p4q.p4q_device_status() == 0
    assert torch.equal(a[5], b[5])
    assert int(a[5].min()) >= 0 and int(a[5].max()) < 1000
    assert torch.equal(a[6].k, b[6].k) and torch.equal(a[6].v, b[6].v) and torch.equal(a[6].lens, b[6].lens)


def test_decode_steps_match_one_prefill(p4q, gen, monkeypatch):
    new = 12
    c, decoder, rows, rot_pos, end, tokens, cache = _run(gen, True, new)
    B, S, _ = rows.shape
    # the prompt and all but the last token at once
    fed = tokens[:, :new - 1]
    x = torch.cat((rows, decoder.embedding[fed.long()]), dim=1)
    at = torch.cat((rot_pos, torch.arange(end, end + new - 1, dtype=torch.int32, device="cuda").expand(B, -1)), dim=1)
    again = gen.Cache(decoder, B, S + new, end + new)
    outs = {"prompt": [], "paged": []}
    prompt, paged = p4q.p4q_causal_attention, p4q.p4q_paged_attention

    def keep_prompt(q, k, v, o, *rest):
        prompt(q, k, v, o, *rest)
        outs["prompt"].append(o)

    def keep_paged(q, k, v, table, lens, o, *rest):
        paged(q, k, v, table, lens, o, *rest)
        outs["paged"].append(o)

    monkeypatch.setattr(p4q, "p4q_causal_attention", keep_prompt)
    monkeypatch.setattr(p4q, "p4q_paged_attention", keep_paged)
    gen.prefill(decoder, again, x.contiguous(), at.contiguous())
    torch.cuda.synchronize()
    assert p4q.p4q_device_status() == 0
    assert torch.equal(cache.lens, again.lens) and torch.equal(cache.table, again.table)
    assert torch.equal(cache.k[0], again.k[0]) and torch.equal(cache.v[0], again.v[0])
    # the last decode step once more, against the prefill's last rows
    cache.lens.sub_(1)
    gen.decode(decoder, cache, fed[:, -1].contiguous(), torch.full((B,), end + new - 2, dtype=torch.int32, device="cuda"))
    o1 = outs["prompt"][0].view(B, S + new - 1, -1)[:, -1].double()
    o2 = outs["paged"][0].double()
    vmax = float(cache.v[0].abs().max())
    bound = 5.2e-4 * (vmax + o1.abs()) + 1e-5 + 2.0 ** -11 * o1.abs() + 1e-4 * vmax
    assert bool(((o1 - o2).abs() <= bound).all()), float(((o1 - o2).abs() / bound).max())


def test_greedy_answers_are_the_largest_logits(p4q, gen):
    zero = torch.zeros((3,), device="cuda")
    c, decoder, rows, rot_pos, end, tokens, cache = _run(gen, False, 2, temperature=zero)
    fresh = gen.Cache(decoder, 3, rows.shape[1] + 2, end + 2)
    logits = gen.prefill(decoder, fresh, rows, rot_pos)
    assert torch.equal(tokens[:, 0].long(), logits.float().argmax(1))
