"""Sizes that 32 bits cannot hold are refused by the binding, not cut to what is left of them."""
import pytest

from paper_2009_13977_amd import binding as B

FAR = 2 ** 32 + 5


@pytest.mark.parametrize("n", [FAR, 2 ** 31, 2 ** 33 + 64, -2 ** 32 + 5, -2 ** 31 - 1])
def test_workspaces(n):
    for ask, args in ((B.fasth_embed_workspace_bytes, (10, 8, 4)), (B.fasth_norm_workspace_bytes, (8, 4)), (B.fasth_log_prob_workspace_bytes, (10, 4, 2))):
        assert ask(*args) > 0
        for at in range(len(args)):
            assert ask(*args[:at], n, *args[at + 1:]) == 0


def test_matrices():
    """Views of one element that are as large as that: the sizes are looked at before anything else."""
    import torch
    tall, wide = torch.zeros(1, 1).expand(FAR, 1), torch.zeros(1, 1).expand(1, FAR)
    t, ids, v = torch.zeros(4, 4), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    calls = (lambda x: B.fasth_embed(x, ids, t), lambda x: B.fasth_embed(t, ids, x), lambda x: B.fasth_embed_backward(ids, t, x, None),
             lambda x: B.fasth_embed_backward(ids, x, t, None), lambda x: B.fasth_norm(x, v, t, v),
             lambda x: B.fasth_norm_backward(x, t, v, v, t, v, None), lambda x: B.fasth_log_prob(x, ids, v, v, t, None),
             lambda x: B.fasth_log_prob(t, ids, v, v, t, None, top_logp=x, top_ids=t),
             lambda x: B.fasth_log_prob_backward(x, ids, t, v, v, v, t))
    for call in calls:
        for x in (tall, wide):
            with pytest.raises(B.FasthError) as e:
                call(x)
            assert e.value.code == B.FASTH_EUNSUPPORTED
