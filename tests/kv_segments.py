"""Long contexts whose results show every token: the values of 16 tokens that follow each other are 1 in one element and 0 elsewhere, the next 16
tokens' in the next element, round and round.  All values being >= 0, an error of the weights is one of the result in the same proportion, so that the bound is
relative to each element: nothing is hidden by values that cancel."""
import numpy as np

from kv_util import EPS32

RUN = 16  # tokens


def elements(length, dim):
    """The element that token j's value sets."""
    return np.arange(length) // RUN % dim


def expected(scores, sees, dim, element=None):
    """softmax of scores [..., L] over what is seen, summed an element at a time: [..., dim], and the number of tokens seen."""
    element = elements(scores.shape[-1], dim) if element is None else element
    z = np.where(sees, scores, -np.inf)
    w = np.where(sees, np.exp(z - z.max(-1, keepdims=True)), 0.0)
    out = np.zeros((*scores.shape[:-1], dim))
    for d in range(dim):
        out[..., d] = w[..., element == d].sum(-1)
    return out / w.sum(-1, keepdims=True), np.broadcast_to(sees, scores.shape).sum(-1)


def misses(got, want, qk, seen, dim, dtype):
    """How far the worst element is outside: a score off by d scales weights and their sum by e^d each, sums of n terms by 1 + 2 n 2^-24,
    rounding to bf16 weights, their sum and the result by 1 + 2^-9 each; at most 1 is within the bound."""
    rel = 2.0 * (dim + 8) * EPS32 * (qk + 1.0) + (seen + 8.0) * 2.0 * EPS32
    if dtype == "bf16":
        rel = rel + 3.0 * 2.0 ** -9
    rel = np.asarray(np.expm1(rel * 1.01))
    return float((np.abs(got - want) / (want * rel[..., None] + 1e-30)).max())
