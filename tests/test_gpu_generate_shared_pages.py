"""Answers that share a prompt share its pages: the cache has one set of them per prompt."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("answers,prompt,most", [(1, 0, 40), (2, 29, 40), (4, 32, 40), (3, 5, 12), (5, 8, 9)])
def test_whole_pages_of_a_prompt_are_the_first_answers_only(p4q, answers, prompt, most):
    from paper_2609_34867_gb300 import generate as gen
    c = gen.Config(d=512, heads=4, kv_heads=2, ffn=1024, layers=2, vocab=1000, page=8)
    prompts, shared, per = 3, prompt // 8, (most + 7) // 8
    cache = gen.Cache(gen.Decoder(c, 3), prompts * answers, most, most, answers=answers, prompt=prompt)
    pages = prompts * (shared + answers * (per - shared))
    assert cache.k.shape[1] == cache.v.shape[1] == pages
    rows = cache.table.view(prompts, answers, per)
    assert bool((rows[:, 1:, :shared] == -1).all())
    own = torch.cat((rows[:, 0, :shared].reshape(-1), rows[:, :, shared:].reshape(-1)))
    assert torch.equal(own.sort().values, torch.arange(pages, dtype=torch.int32, device=own.device))


@pytest.mark.parametrize("answers", [1, 3])
def test_answers_do_not_depend_on_the_pages(p4q, answers):
    """Each prompt's answers are those that a cache with another order of pages gives."""
    from paper_2609_34867_gb300 import generate as gen
    c = gen.Config(d=512, heads=4, kv_heads=2, ffn=1024, layers=2, vocab=1000, page=8)
    decoder = gen.Decoder(c, 3)
    rows, rot_pos, end = gen.pruned_prompt(2, c, 5, N=96, K=24, T=5)
    n, new, S = 2 * answers, 12, rows.shape[1]
    logits = []
    for seed in (0, 7):
        cache = gen.Cache(decoder, n, S + new, end + new, seed=seed, answers=answers, prompt=S)
        last = gen.prefill(decoder, cache, rows, rot_pos).repeat_interleave(answers, 0)
        at = torch.full((n,), end, dtype=torch.int32, device="cuda")
        got = [last]
        for i in range(new - 1):
            token = torch.arange(n, dtype=torch.int32, device="cuda") * 7 + i
            got.append(gen.decode(decoder, cache, token, at))
            at.add_(1)
        torch.cuda.synchronize()
        assert p4q.p4q_device_status() == 0
        logits.append(torch.stack(got))
    assert torch.equal(*logits)
