"""The recurrent language model of examples/: its gradients against autograd on
the plain formulas in 64 bits, its one-token form against the whole sequence,
and that it learns."""

import importlib.util
import os

import pytest
import torch

from paper_1709_02755_amd import sru

pytestmark = pytest.mark.gpu

# Float32 throughout: a product or an operator adds at most 1e-5 of the norm of
# its result (the bound of this library's float32 checks); forward and backward
# of two blocks are about 20 of them in a row, and the norms and the softmax of
# these inputs amplify a relative error by less than 5: 20 * 5 * 1e-5.
TOL = 1e-3

_spec = importlib.util.spec_from_file_location("recurrent_lm", os.path.join(
    os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "recurrent_lm.py"))
example = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(example)


def far(got, ref):
    return float((got.double().cpu() - ref).norm() / ref.norm())


def plain(p, tokens, blocks):
    """Logits [L * B, V] by the formulas, in the type of the parameters."""
    L, B = tokens.shape

    def norm(v):
        return v / torch.sqrt(v.square().mean(-1, keepdim=True) + 1e-6)

    x = p["embed"][tokens]
    o = norm(x) * p["pre0"]
    for n in range(blocks):
        v, r, i, z = (o @ p[f"proj{n}"].t()).chunk(4, -1)
        a = torch.exp(-8.0 * torch.nn.functional.softplus(p[f"lam{n}"]) * torch.sigmoid(r))
        h, H = torch.zeros_like(x[0]), []
        for t in range(L):
            new = (tokens[t] == 0).unsqueeze(1)
            at = torch.where(new, torch.zeros_like(a[t]), a[t])
            h = at * h + torch.sqrt(1 - at * at) * torch.sigmoid(i[t]) * v[t]
            H.append(h)
        y = norm(torch.stack(H)) * p[f"post{n}"] * torch.nn.functional.silu(z)
        x = x + p[f"scale{n}"] * y
        o = norm(x) * p[f"pre{n + 1}"]
    return (o @ p["head"].t()).reshape(L * B, -1)


@pytest.mark.parametrize("width,vocab,L,B", [(64, 200, 9, 3), (40, 77, 70, 2), (128, 301, 130, 1)])
def test_gradients_and_loss(width, vocab, L, B):
    dev = torch.device("cuda:0")
    m = example.RecurrentLM(vocab, width, 2, dev, gemm_dtype=sru.GEMM_FP32)
    tokens, targets, ids, tl = example.Source(vocab, 5, dev).batch(L, B)
    p = {n: t.double().cpu().requires_grad_() for n, t in m.p.items()}
    z = plain(p, tokens.cpu(), 2)
    N = L * B

    logp = z.log_softmax(1)
    loss = -logp.gather(1, targets.cpu().reshape(-1, 1)).mean()
    ref = dict(zip(p, torch.autograd.grad(loss, p.values(), retain_graph=True)))
    got, grads = m.fit(tokens, targets)
    assert abs(float(got) - loss.item()) <= TOL * loss.item()
    for n in p:
        assert far(grads[n], ref[n]) <= TOL, n

    q = tl.double().cpu().log_softmax(1)
    kl = (q.exp() * (q - logp.gather(1, ids.cpu()))).sum() / N
    ref = dict(zip(p, torch.autograd.grad(kl, p.values())))
    got, grads = m.distill(tokens, ids, tl)
    assert abs(float(got) - kl.item()) <= TOL * kl.item()
    for n in p:
        assert far(grads[n], ref[n]) <= TOL, n


# With bfloat16 activations every tensor between the operators is rounded, by at
# most 2^-8 of its values: o, u and H of two blocks and the logits forward, dlogits
# and do, dy and du of two blocks back, 14 of them; times the 5 of above.
TOL_BF16 = 14 * 5 * 2.0 ** -8


@pytest.mark.parametrize("width,vocab,L,B", [(64, 200, 9, 3), (40, 77, 70, 2)])
def test_gradients_and_loss_with_bfloat16_activations(width, vocab, L, B):
    dev = torch.device("cuda:0")
    m = example.RecurrentLM(vocab, width, 2, dev, gemm_dtype=sru.GEMM_FP32, act=torch.bfloat16)
    tokens, targets, ids, tl = example.Source(vocab, 5, dev).batch(L, B)
    p = {n: t.double().cpu().requires_grad_() for n, t in m.p.items()}
    logp = plain(p, tokens.cpu(), 2).log_softmax(1)
    loss = -logp.gather(1, targets.cpu().reshape(-1, 1)).mean()
    q = tl.double().cpu().log_softmax(1)
    kl = (q.exp() * (q - logp.gather(1, ids.cpu()))).sum() / (L * B)
    for of, (got, grads) in ((loss, m.fit(tokens, targets)), (kl, m.distill(tokens, ids, tl))):
        ref = dict(zip(p, torch.autograd.grad(of, p.values(), retain_graph=True)))
        assert abs(float(got) - of.item()) <= TOL_BF16 * of.item()
        for n in p:
            assert far(grads[n], ref[n]) <= TOL_BF16, n
    state = m.new_state(B)
    steps = torch.stack([m.step(tokens[t], state) for t in range(L)])
    assert steps.dtype == torch.bfloat16
    whole = m.forward(tokens)[0].view(L, B, vocab)
    assert far(steps, whole.double().cpu()) <= TOL_BF16


def test_one_token_at_a_time_and_in_pieces():
    dev, L, B, V = torch.device("cuda:0"), 37, 5, 130
    m = example.RecurrentLM(V, 96, 2, dev, gemm_dtype=sru.GEMM_FP32)
    tokens = example.Source(V, 4, dev).batch(L, B)[0]
    whole = m.forward(tokens)[0].view(L, B, V)
    state = m.new_state(B)
    steps = torch.stack([m.step(tokens[t], state) for t in range(L)])
    assert far(steps, whole.double().cpu()) <= TOL
    part = m.new_state(B)
    pieces = torch.cat([m.forward(tokens[a:b].contiguous(), part)[0].view(-1, B, V)
                        for a, b in ((0, 1), (1, 20), (20, L))])
    assert far(pieces, whole.double().cpu()) <= TOL
    for a, b in zip(state, part):
        assert far(a, b.double().cpu()) <= TOL


def test_it_learns_and_speaks():
    dev, V, L, B = torch.device("cuda:0"), 256, 64, 16
    m = example.RecurrentLM(V, 64, 2, dev)
    source = example.Source(V, 8, dev)
    opt = torch.optim.Adam(m.p.values(), lr=3e-3)
    losses = []
    for _ in range(40):
        tokens, targets, ids, tl = source.batch(L, B)
        loss, grads = m.distill(tokens, ids, tl)
        for n, t in m.p.items():
            t.grad = grads[n]
        opt.step()
        losses.append(float(loss))
    assert losses[-1] < 0.5 * losses[0], losses
    said, logps = m.generate(torch.zeros(3, dtype=torch.int64, device=dev), 7, m.new_state(3), top=8)
    assert said.shape == (7, 3) and int(said.min()) >= 0 and int(said.max()) < V
    # the same tokens, scored as a sequence
    before = torch.cat([torch.zeros_like(said[:1]), said[:-1]])
    again = m.score(before, said, top=8)
    # bfloat16 products of another row count add in another order
    assert torch.allclose(again["logprob"].view(7, 3), logps, atol=5e-2)
