"""The synthetic text of the recurrent language model's example, on the CPU."""

import importlib.util
import os

import torch

_spec = importlib.util.spec_from_file_location("recurrent_lm", os.path.join(
    os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "recurrent_lm.py"))
example = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(example)


def test_a_token_that_follows_more_than_once_counts_as_all():
    """What the source itself gives its text, against its transition matrix."""
    V, fan, L, B = 5, 16, 30, 4
    source = example.Source(V, fan, "cpu")
    tokens, targets, ids, logits = source.batch(L, B)
    matrix = torch.zeros(V, V, dtype=torch.float64)
    matrix.scatter_add_(1, source.ids, source.logits.double().softmax(1))
    assert torch.allclose(matrix.sum(1), torch.ones(V, dtype=torch.float64))
    want = torch.log(matrix[tokens.reshape(-1), targets.reshape(-1)])
    got = source.logprobs(targets.reshape(-1), ids, logits)
    # fp32: a few roundings of 2^-24 of values up to 20
    assert got.shape == want.shape and float((got.double() - want).abs().max()) <= 1e-5
