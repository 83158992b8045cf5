"""Generation with a cache of 8 or 4 bits, and with answers that share a prompt: the calls of
append and attention together, as a decode loop makes them.

Layer 0's keys and values do not depend on attention (the integer linears are exact), so a
cache of codes has there what the 16-bit cache has, within half a step of the scale and the
roundings to fp16 of the two rotations (one of them 2^-11, in the other another 2^-22). The
attention of shared prompts is compared with the formula in 64 bits on what the cache holds:
2^-11 |o| + 1e-4 vmax, as for the attention over a cache of one's own."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gen(p4q):
    from paper_2609_34867_gb300 import generate
    return generate


def _run(gen, graph, new=10, B=3, answers=1, bits=16, **params):
    c = gen.Config(d=512, heads=4, kv_heads=2, ffn=1024, layers=2, vocab=1000, page=8)
    decoder = gen.Decoder(c, 3)
    rows, rot_pos, end = gen.pruned_prompt(B, c, 5, N=96, K=24, T=5)
    u = torch.rand((new, B * answers), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    tokens, _, cache = gen.generate(decoder, rows, rot_pos, end, new, u, graph=graph, bits=bits, answers=answers, **params)
    return c, tokens, cache, rows.shape[1]


@pytest.mark.parametrize("bits", [8, 4])
def test_codes_hold_what_16_bits_hold(p4q, gen, bits):
    c, _, full, S = _run(gen, True, new=1)
    _, tokens, codes, _ = _run(gen, True, new=1, bits=bits)
    assert p4q.p4q_device_status() == 0
    assert torch.equal(full.table, codes.table)
    seqs = full.table.shape[0]
    j = torch.arange(S, device="cuda")
    at = full.table.long()[:, j // c.page], j % c.page
    for a, b, s in ((full.k, codes.k, codes.k_scale), (full.v, codes.v, codes.v_scale)):
        x, q, scale = a[0][at].double(), b[0][at], s[0][at].double()[..., None]
        if bits == 4:
            w = torch.stack((q & 15, q >> 4), -1).flatten(-2).to(torch.int16)
            q = torch.where(w > 7, w - 16, w)
        assert x.shape == (seqs, S, c.kv_heads, 128)
        bound = scale * 0.5 * (1 + 2.0 ** -20) + (2.0 ** -10 + 2.0 ** -20) * x.abs() + 2.0 ** -24
        assert bool(((q.double() * scale - x).abs() <= bound).all())


@pytest.mark.parametrize("bits,answers", [(8, 1), (4, 1), (16, 4)])
def test_steps_and_their_graph_give_the_same_tokens(p4q, gen, bits, answers):
    p = torch.full((3 * answers,), 0.9, device="cuda")
    a = _run(gen, False, bits=bits, answers=answers, top_p=p)
    b = _run(gen, True, bits=bits, answers=answers, top_p=p)
    assert p4q.p4q_device_status() == 0
    assert torch.equal(a[1], b[1]) and int(a[1].min()) >= 0 and int(a[1].max()) < 1000
    assert torch.equal(a[2].k, b[2].k) and torch.equal(a[2].v, b[2].v) and torch.equal(a[2].lens, b[2].lens)


@pytest.mark.parametrize("answers", [2, 5])
def test_answers_see_the_prompt_and_their_own_tokens(p4q, gen, monkeypatch, answers):
    seen = []
    real = p4q.p4q_prefix_attention

    def keep(q, k, v, table, lens, start, prefix, o, ws, **more):
        real(q, k, v, table, lens, start, prefix, o, ws, **more)
        if not torch.cuda.is_current_stream_capturing():
            seen.append((q.clone(), k.clone(), v.clone(), lens.clone(), o.clone()))

    monkeypatch.setattr(p4q, "p4q_prefix_attention", keep)
    c, tokens, cache, S = _run(gen, False, new=6, answers=answers)
    assert p4q.p4q_device_status() == 0 and len(seen) == 5 * c.layers
    n = tokens.shape[0]
    assert n == 3 * answers and torch.equal(cache.lens, torch.full_like(cache.lens, S + 5))
    for q, k, v, lens, o in seen:
        for b in range(n):
            j = torch.arange(int(lens[b]), device="cuda")
            row = torch.where(j < S, b // answers * answers, b)
            pg = cache.table.long()[row, j // c.page]
            kk, vv = (x[pg, j % c.page].double().repeat_interleave(c.heads // c.kv_heads, 1) for x in (k, v))
            s = torch.einsum("hd,lhd->hl", q[b].double().view(c.heads, 128), kk) / 128 ** 0.5
            want = torch.einsum("hl,lhd->hd", torch.softmax(s, -1), vv)
            err = (o[b].double().view(c.heads, 128) - want).abs()
            assert bool((err <= 2.0 ** -11 * want.abs() + 1e-4 * vv.abs().max()).all())


def test_greedy_answers_to_one_prompt_are_one_answer(p4q, gen):
    zero = torch.zeros((12,), device="cuda")
    _, tokens, _, _ = _run(gen, True, answers=4, temperature=zero)
    assert torch.equal(tokens.view(3, 4, -1), tokens.view(3, 4, -1)[:, :1].expand(3, 4, -1))


def test_codes_and_shared_prompts_do_not_go_together(p4q, gen):
    with pytest.raises(ValueError):
        _run(gen, False, bits=8, answers=2)
    with pytest.raises(SystemExit):
        gen.main(["--answers", "2", "--cache-bits", "4"])


def test_the_command_runs(p4q, gen, capsys):
    for argv in (["--cache-bits", "4"], ["--answers", "3"]):
        assert gen.main(["--images", "2", "--new", "4", *argv]) == 0
    out = capsys.readouterr().out
    assert out.count("image 0:") == 4 and "us per decode step of 6 sequences" in out
