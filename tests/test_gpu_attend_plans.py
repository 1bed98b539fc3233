"""Plans that do not belong to the call that meets them: of another cache, of an earlier owner of the workspace's memory."""
import pytest
import torch

from paper_2601_07667_b200 import binding as B

from pages_check import Both, check_attention, ints

pytestmark = pytest.mark.gpu


def left_alone(cache, batch, heads):
    out = torch.full((batch.n_tokens, heads, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((batch.n_tokens, heads), 7.0, device="cuda")
    cache.attend(0, batch, torch.ones_like(out), out, lse)
    assert B.asl_pages_status(cache.ctx, cache.pages) == (B.ASL_ERR_WORKSPACE, -1)
    assert (out == 7.0).all() and (lse == 7.0).all()


def forked(**sizes):
    """A prompt of 90 tokens in the last slots but five and five forks of it behind it."""
    both = Both(kv_heads=2, **sizes)
    n = sizes["max_seqs"]
    both.fill([0] * (n - 6) + [90] + [0] * 5)
    both.fork([-1] * (n - 6) + [-1] + [n - 6] * 5)
    both.fill([-1] * (n - 5) + [91, 95, 99, 100, 92])
    return both


@pytest.mark.parametrize("share", [0, 2])
@pytest.mark.parametrize("other", [dict(page=64), dict(max_seqs=7), dict(max_pages=8), dict()])
def test_a_plan_of_another_cache_is_refused(other, share):
    """The plan names slots that the other cache's table may not have, and prefixes of whole pages of another size: refused by
    what differs, or, where all sizes agree, by the table that it was made from."""
    sizes = dict(page=16, n_pages=80, max_seqs=40, max_pages=12)
    a, b = forked(**sizes), forked(**{**sizes, **other})
    batch = a.cache.batch(ints(range(34, 40)), ints(range(7)), n_tokens=6, n_q_heads=8)
    a.cache.plan(batch, share=share)
    left_alone(b.cache, batch, 8)
    n = b.cache.len.numel()
    check_attention(b, 0, list(range(n - 6, n)), list(range(7)), 8, share=share)
    check_attention(a, 0, list(range(34, 40)), list(range(7)), 8, share=share)


def test_a_batch_may_serve_several_caches():
    """Rows appended and attention planned anew for each of two caches with the same slots."""
    sizes = dict(page=16, n_pages=80, max_seqs=40, max_pages=12)
    a, b = forked(**sizes), forked(**sizes, seed=1)
    batch = a.cache.batch(ints(range(34, 40)), ints(range(7)), n_tokens=6, n_q_heads=8)
    q = torch.randn((6, 8, 128), device="cuda").to(torch.bfloat16)
    for both in (a, b):
        both.cache.plan(batch, share=2)
        out = both.cache.attend(0, batch, q)
        both.cache.check()
        o, _, tol, _ = both.expect(0, list(range(34, 40)), list(range(7)), q.double().cpu().numpy(), 8)
        assert (abs(out.double().cpu().numpy() - o) <= tol).all()


def test_a_plan_that_an_earlier_batch_left_is_none():
    """A batch whose workspace lies where another's did, plan and all."""
    both = forked(page=16, n_pages=80, max_seqs=40, max_pages=12)
    slots, cu = ints(range(34, 40)), ints(range(7))
    batch = both.cache.batch(slots, cu, n_tokens=6, n_q_heads=8)
    both.cache.plan(batch)
    at = batch.ws
    del batch
    batch = both.cache.batch(slots, cu, n_tokens=6, n_q_heads=8)
    assert batch.ws == at
    left_alone(both.cache, batch, 8)
