"""Drafted trees of a stack that serves longer prompts than a tree may have nodes: the
width of the trees' bits says how many nodes a request has at most."""
import pytest
import torch

import synth
from tests import test_gpu_tree_attention as tree_test
from tests.test_gpu_attention_stack import DIM, HEADS, HIDDEN, KV, PAGE, Served, _pass, _stack

pytestmark = pytest.mark.gpu


class Narrow(tree_test.Tree):
    """Bits of `words` words, whatever the stack's bound."""
    words = 1

    def bits(self, words):
        return super().bits(self.words)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("nodes,words", [([13, 64, 1], 1), ([13, 64, 1], 3), ([65, 2, 100], 2),
                                         ([3, 200, 0], 4)])
def test_trees_behind_long_prompts(nodes, words, dt):
    table = torch.randperm(3 * 60, generator=torch.Generator().manual_seed(6)).int().reshape(3, 60)
    s = _stack(300, 3, 60, 181, dt)
    ids = torch.randint(-1, 5, (300,), generator=torch.Generator().manual_seed(7)).int().cuda()
    x = lambda i: synth.normal((300, HIDDEN), dt, 9900 + i).cuda()
    rows = [280, 3, 17]
    _pass(s, Served(s, rows, rows, table, dt), dt, x(0), ids)
    tree = Narrow(nodes, rows, HEADS, KV, DIM, PAGE, dt, seed=9)
    tree.tokens, tree.words = s.tokens, words
    _pass(s, Served(s, nodes, [n + c for n, c in zip(nodes, rows)], table, dt), dt, x(1), ids, tree)
    # and the accepted ones
    keep = torch.tensor([[0, 1], [0, -1], [0, -1]], dtype=torch.int32).cuda()
    kept = torch.tensor([2, 1, 0], dtype=torch.int32).cuda()
    b = Served(s, nodes, [n + c for n, c in zip(nodes, rows)], table, dt)
    s.keep(b.gpu(), keep, kept)


def test_refuses_bits_of_other_widths():
    from paper_2511_19457_amd.abi import SparoaError
    s = _stack(300, 2, 60, 121, "bf16")
    x = torch.zeros(300, HIDDEN).bfloat16().cuda()
    i = lambda *n: torch.zeros(*n, dtype=torch.int32).cuda()
    for bits in (torch.zeros(300, 5), torch.zeros(300, 0), torch.zeros(299, 1), torch.zeros(301, 1)):
        with pytest.raises((SparoaError, ValueError)):
            s.forward(x, i(300), batch=(i(3), i(2), i(2, 60)), tree=(bits.long().cuda(), i(300)))
