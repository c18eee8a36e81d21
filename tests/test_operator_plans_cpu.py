"""Plans of the operators beside the path as objects of a model: copied, pickled, saved."""
import copy
import dataclasses
import io
import pickle

import pytest
import torch

import paper_2604_20368_b200 as ln


def _through_torch(x):
    f = io.BytesIO()
    torch.save(x, f)
    f.seek(0)
    return torch.load(f, weights_only=False)


WAYS = [copy.copy, copy.deepcopy, lambda x: pickle.loads(pickle.dumps(x)), _through_torch]


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("freq", [None, [1.0, 0.5, 0.25, -0.125]])
def test_rope_survives_copies(way, freq):
    rope = ln.Rope(64, freq, interleaved=True, factor=1.5)
    other = way(rope)
    assert (other.d, other.r, other.interleaved, other.factor) == (64, 0 if freq is None else 8, True, 1.5)
    assert other.turns is None if freq is None else torch.equal(other.turns, rope.turns)
    assert type(other.plan) is type(rope.plan) and other.plan is not rope.plan
    with pytest.raises(ValueError, match="CUDA"):               # the plan is one that the entry points take
        ln.rope_fwd(other, torch.zeros(1, 1, 2, 64))


@pytest.mark.parametrize("way", WAYS)
def test_softmax_attention_survives_copies(way):
    sp = ln.SoftmaxAttention(scale=0.25, cap=20.0, causal=True, kv_len=torch.tensor([3, 5], dtype=torch.int32))
    other = way(sp)
    assert (other.scale, other.cap, other.causal, other.prefix) == (0.25, 20.0, True, None)
    assert torch.equal(other.kv_len, sp.kv_len) and other.plan is not sp.plan
    x = torch.zeros(2, 1, 4, 32)
    with pytest.raises(ValueError, match="CUDA"):
        ln.softmax_attention_fwd(other, x, x, x)
    with pytest.raises(dataclasses.FrozenInstanceError):
        other.cap = 1.0


def test_a_model_that_holds_plans_is_copied_whole():
    class Layer(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.w = torch.nn.Parameter(torch.ones(3))
            self.rope, self.attention = ln.Rope(32, [1.0] * 8), ln.SoftmaxAttention(causal=True)

    layer = Layer()
    other = copy.deepcopy(layer)
    assert torch.equal(other.rope.turns, layer.rope.turns) and other.rope.turns.data_ptr() != layer.rope.turns.data_ptr()
    assert other.attention.causal


@pytest.mark.filterwarnings("error")
def test_a_frequency_just_below_zero_is_a_whole_turn():
    """-1e-30 radians are 1 - 1.6e-31 turns, which the 64 bits of the table's arithmetic round to one turn: the fraction is 0 or 2^64 - 1."""
    rope = ln.Rope(64, [-1e-30, -1e-19, 1e-30, -0.25, 0.25])
    t = [x % 2 ** 64 for x in rope.turns.tolist()]
    assert min(t[0], 2 ** 64 - t[0]) <= 1 and min(t[1], 2 ** 64 - t[1]) <= 1 and t[2] == 0
    assert abs((t[3] + t[4]) - 2 ** 64) <= 1
