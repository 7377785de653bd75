"""What token_logprob returns is a named tuple of four, to unpack and to torch's trees, with room for what the way back needs."""
import copy
import pickle

import torch
from torch.utils import _pytree as tree

import paper_2203_16340_amd as L


def _one():
    r = L.TokenLogprob(torch.zeros(2), torch.ones(2), torch.full((2,), 2.0), None)
    r.stats = torch.arange(4.0).view(2, 2)
    return r


def test_a_tuple_of_four():
    r = _one()
    logp, lse, lse_rest, entropy = r
    assert len(r) == 4 and isinstance(r, tuple) and r._fields == ("logp", "lse", "lse_rest", "entropy")
    assert logp is r.logp and lse is r[1] and lse_rest is r.lse_rest and entropy is None
    assert list(r._asdict()) == list(r._fields) and "TokenLogprob(logp=" in repr(r)


def test_trees_reach_its_tensors():
    r = _one()
    assert len(tree.tree_leaves(r)) == 4
    twice = tree.tree_map(lambda t: t if t is None else 2 * t, r)
    assert type(twice) is L.TokenLogprob and torch.equal(twice.lse, 2 * r.lse) and twice.stats is None


def test_put_together_again():
    r = _one()
    assert L.TokenLogprob(*r).stats is None and r._replace(entropy=r.logp).stats is None
    for q in (copy.copy(r), pickle.loads(pickle.dumps(r))):
        assert type(q) is L.TokenLogprob and torch.equal(q.stats, r.stats) and torch.equal(q.lse, r.lse)
