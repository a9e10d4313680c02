"""The 64-bit definitions of a cache in four bits and of normed, rotated heads (oracle/star_q4.py) against values by hand."""
import math

import torch

from oracle import star_q4


def _group(*first):
    return torch.tensor(list(first) + [0.0] * (32 - len(first)))[None]


def test_codes_and_units():
    codes, e = star_q4.quantise(_group(6.0, -0.25, 0.75, 2.5, -5.0, 0.26, 1.25, -0.0))
    assert e.tolist() == [[127]]
    assert codes[0, :4].tolist() == [7 + 16 * 8, 2 + 16 * 4, (6 + 8) + 16 * 1, 2 + 16 * 8]       # ties to the even code, signs kept
    assert star_q4.values(codes, e)[0, :8].tolist() == [6, -0.0, 1, 2, -4, 0.5, 1, -0.0]


def test_largest_element_decides():
    for most, unit in ((3.5, 0), (6.99, 0), (7.0, 1), (3.49, -1), (1.0, -2), (1.75, -1), (1.7499, -2)):
        assert star_q4.quantise(_group(most))[1].item() == 127 + unit, most
    assert star_q4.quantise(_group(0.0))[1].item() == 127 and star_q4.quantise(_group(-0.0, 0.0))[1].item() == 127
    assert star_q4.quantise(_group(1e-40))[1].item() == 2
    codes, e = star_q4.quantise(_group(3.4e38))
    assert e.item() == 252 and star_q4.values(codes, e)[0, 0].item() == 6 * 2.0 ** 125


def test_what_is_not_finite_marks_its_group():
    x = torch.ones(1, 96)
    x[0, 40], x[0, 70] = math.inf, math.nan
    codes, e = star_q4.quantise(x)
    assert e.tolist() == [[125, 255, 255]] and star_q4.values(codes, e).isnan().sum() == 64


def test_error_of_a_group():
    x = torch.randn(4000, 64, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    v = star_q4.values(*star_q4.quantise(x))
    most = x.unflatten(-1, (2, 32)).abs().amax(-1, keepdim=True)
    off = (v - x).unflatten(-1, (2, 32)).abs()
    # one unit between 4 and 6 of them, which only a group whose largest is 5 or more comes to (most - 4 below); half a unit from 2 on
    assert (off <= most / 5 + 1e-12).all() and (off > most / 6).any()


def test_attention_of_two_keys():
    Q = torch.tensor([[2.0, 0.0], [0.0, 1.0]])
    K, V = torch.tensor([[1.0, 0.0], [0.0, 3.0]]), torch.tensor([[1.0, 0.0], [0.0, 1.0]])
    A, lse, size, most, total = star_q4.attend(Q, K, V, 0.5, cache_len=0)
    assert torch.allclose(A[0], torch.tensor([1.0, 0.0]).double()) and lse[0].item() == 1.0            # the first sees itself alone
    w = torch.softmax(torch.tensor([0.0, 1.5]).double(), 0)
    assert torch.allclose(A[1], w) and torch.allclose(size[1], w) and most.tolist() == [1.0, 1.5]
    assert total.tolist() == [[1.0, 0.0], [1.0, 1.0]]


def test_norm_and_rotation_by_hand():
    x = torch.zeros(1, 1, 1, 4)
    x[..., 0], x[..., 2], x[..., 1] = 3.0, 4.0, 5.0
    w = torch.tensor([1.0, 2.0, 1.0, 1.0])
    y, _ = star_q4.norm_rope(x, w, 0.0, 100.0, torch.tensor([[[1, 7]]]), [0, 1])
    r = 1 / math.sqrt(50 / 4)
    want = [r * (3 * math.cos(1) - 4 * math.sin(1)), 10 * r * math.cos(0.7), r * (4 * math.cos(1) + 3 * math.sin(1)), 10 * r * math.sin(0.7)]
    assert torch.allclose(y.flatten(), torch.tensor(want, dtype=torch.float64))
    y, _ = star_q4.norm_rope(x, None, 0.0, 100.0, torch.tensor([[[0, 0]]]), [0, 1])
    assert torch.equal(y, x.double())
