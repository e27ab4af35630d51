"""The serving example with fewer pages than its requests want: who is refused brings the same tokens again, and loses none."""
import pytest
import torch

from test_gpu_kv_serving import example, free

pytestmark = pytest.mark.gpu

VOCAB = 1000


class Successor:
    """A model whose next token follows from the last one and its position alone."""
    layers, kv_heads, head_dim = 1, 1, 64

    def __init__(self):
        self.refusals = 0

    def forward(self, kv, tokens, max_new):
        self.refusals += kv.refused.item()
        return torch.nn.functional.one_hot((7 * tokens + kv.position[:len(tokens)] + 3) % VOCAB, VOCAB).float()


def expected(prompt, n):
    tokens = list(prompt)
    for _ in range(n):
        tokens.append((7 * tokens[-1] + len(tokens) - 1 + 3) % VOCAB)
    return tokens[len(prompt):]


@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
@pytest.mark.parametrize("pages", (4, 5, 7, None))
def test_refused_requests_wait(gpu_device, pages, window, sinks):
    prompts, steps = [[1, 2, 3], list(range(30)), [7] * 17, [9, 8]], 12
    model = Successor()
    made, kv = example().serve(model, prompts, steps, window, sinks, pages)
    assert made == [expected(p, steps - r) for r, p in enumerate(prompts)]
    assert free(kv) == list(range(kv.desc.pages)) and kv.length[0].tolist() == [0] * 4
    assert (model.refusals > 0) == (pages in (4, 5))  # 1 + 3 + 2 + 1 pages hold all


def test_too_few_pages_for_any(gpu_device):
    with pytest.raises(RuntimeError):
        example().serve(Successor(), [list(range(50))], 4, pages=3)
