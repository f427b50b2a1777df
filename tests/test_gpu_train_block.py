"""The example that runs the training-step operators and the optimizer together."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("train_block", os.path.join(ROOT, "examples", "train_block.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_it_learns():
    """The loss starts at the uniform guess's, ln 1000, and the tokens' successors are learnt."""
    print("[gpu-case] train_block", flush=True)
    losses = _example().train(100, say=None)
    assert 6.5 < losses[0] < 8.0 and losses[-1] < 0.5 * losses[0], losses[::10]


def test_its_gradients_are_autograds():
    """One backward pass against the same model in torch's own operations. Inputs held in 8
    bits (3 mantissa bits: 2^-4 of a value at most, 2^-5.8 in the mean square) and bf16
    roundings on other paths leave the directions within a few percent."""
    import torch
    ex = _example()
    block = ex.Block(3)
    tokens = ex.Walks(4).batch()
    loss = block.loss(tokens)
    loss.backward()
    loss = loss.detach()

    class Plain(ex.Block):
        def linear(self, name, x):
            return x @ self.weights[name].t()

        def embed(self, tokens):
            return self.table[tokens] * ex.math.sqrt(ex.WIDTH)

        def norm_rope(self, q, k):
            out = []
            for x, w in ((q, self.gains[0]), (k, self.gains[1])):
                x = x.float()
                z = x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + ex.EPS) * w
                a, b = z.chunk(2, -1)
                c, s = self.cos[None, :, None], self.sin[None, :, None]
                out.append(torch.cat([a * c - b * s, b * c + a * s], -1).bfloat16())
            return out

    plain = Plain(3)
    for w in plain.weights.values():
        w.requires_grad_()
    want = plain.loss(tokens)
    want.backward()
    want = want.detach()
    assert abs(float(loss - want)) < 2e-2 * float(want)
    pairs = [(block.grads[n], plain.weights[n].grad) for n in block.grads]
    pairs += [(block.table.grad, plain.table.grad)] + [(a.grad, b.grad) for a, b in zip(block.gains, plain.gains)]
    for got, ref in pairs:
        got, ref = got.double().flatten(), ref.double().flatten()
        assert float(got @ ref / (got.norm() * ref.norm())) > 0.99
        assert abs(float(got.norm() / ref.norm()) - 1) < 0.05
