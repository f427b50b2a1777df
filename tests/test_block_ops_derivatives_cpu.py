"""Calls that would lose a derivative without a word are refused: tensors that carry a tangent
(the operators have no forward-mode rules), and numbers that are tensors which ask for a gradient. The
refusal comes before any other check, so that it is seen without a GPU."""
import pytest

torch = pytest.importorskip("torch")
import torch.autograd.forward_ad as fwd

import paper_2606_27216_amd as hm

X, W, T = torch.zeros(4, 8), torch.ones(8), torch.zeros(4, dtype=torch.int64)
Q, L = torch.zeros(1, 4, 2, 8), torch.zeros(1, 4, 2)
C = torch.zeros(4, 4)
R = torch.zeros(4)

# (a call, the places of its tensors that a derivative reaches)
CALLS = {
    "embed": ([T, X], [1]),
    "embed_grad": ([T, X, 4], [1]),
    "qk_norm_rope": ([Q, Q, W, W, C, C], [0, 1, 2, 3, 4, 5]),
    "qk_norm_rope_grad": ([Q, Q, Q, Q, W, W, C, C], list(range(8))),
    "add_norm": ([X, X, W], [0, 1, 2]),
    "add_norm_grad": ([X, X, W, X], [0, 1, 2, 3]),
    "attention": ([Q, Q, Q], [0, 1, 2]),
    "attention_grad": ([Q, Q, Q, Q, Q, L], list(range(6))),
    "token_logprob": ([X, T], [0]),
    "token_logprob_grad": ([R, R, X, T, R, R], [0, 1, 2, 4, 5]),
}


@pytest.mark.parametrize("name,place", [(n, p) for n, (_, places) in CALLS.items() for p in places])
def test_tangents_are_refused(name, place):
    args = list(CALLS[name][0])
    with fwd.dual_level():
        with pytest.raises(ValueError):  # (a CPU tensor: refused as before)
            getattr(hm, name)(*args)
        args[place] = fwd.make_dual(args[place], torch.ones_like(args[place]))
        with pytest.raises(NotImplementedError, match=name):
            getattr(hm, name)(*args)
        with torch.no_grad(), pytest.raises(NotImplementedError, match=name):
            getattr(hm, name)(*args)


NUMBERS = [("embed", "scale"), ("embed_grad", "scale"), ("qk_norm_rope", "eps"), ("qk_norm_rope_grad", "eps"), ("add_norm", "eps"),
           ("add_norm_grad", "eps"), ("attention", "scale"), ("attention_grad", "scale"), ("token_logprob", "scale"),
           ("token_logprob_grad", "scale")]


@pytest.mark.parametrize("name,what", NUMBERS)
def test_numbers_that_ask_for_a_gradient_are_refused(name, what):
    args = CALLS[name][0]
    number = torch.tensor(0.5, requires_grad=True)
    with pytest.raises(NotImplementedError, match=name):
        getattr(hm, name)(*args, **{what: number})
    for plain in (number.detach(), 0.5, 1):
        with pytest.raises(ValueError):  # (a CPU tensor: refused as before)
            getattr(hm, name)(*args, **{what: plain})
    with torch.no_grad(), pytest.raises(ValueError):
        getattr(hm, name)(*args, **{what: number})
    with fwd.dual_level(), pytest.raises(NotImplementedError, match=name):
        getattr(hm, name)(*args, **{what: fwd.make_dual(torch.tensor(0.5), torch.tensor(1.0))})
