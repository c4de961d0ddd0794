"""The binding takes a layer's arrays in the documented shape, or with neighbouring dimensions of it joined, and nothing else: the same
number of values in another order would be another layer.  (On the CPU: what passes the checks of shapes is refused for its device.)"""
import pytest
import torch

from paper_2311_15806_b200 import binding as B

E, O, I, G = 3, 40, 256, 64
BF16, U8, I32 = torch.bfloat16, torch.uint8, torch.int32


def _layer(E=E, asymmetric=True, **other):
    d = B.make_group_desc(O, I, G, asymmetric=asymmetric, experts=E)
    a = dict(codes=torch.zeros((E, I // 32, O, 16), dtype=U8), scales=torch.zeros((E, I // G, O), dtype=BF16), zeros=torch.zeros((E, I // G, O), dtype=U8))
    a.update(other)
    return d, a["codes"], a["scales"], a["zeros"]


def _calls(layer, bias):
    E = layer[0].experts
    x, y = torch.zeros((5, I), dtype=BF16), torch.zeros((5, O), dtype=BF16)
    yield lambda: B.pipe_expert_linear(*layer, x, torch.zeros(E + 1, dtype=I32), y, bias=bias)
    if E == 1:
        yield lambda: B.pipe_group_linear(*layer, x, y, bias=bias)
    if bias is None:
        yield lambda: B.pipe_group_quantize(layer[0], torch.zeros((E, O, I)), *layer[1:])


def _refuses(layer, what, bias=None):
    for call in _calls(layer, bias):
        with pytest.raises(B.PipeError, match=what) as e:
            call()
        assert e.value.status == B.PIPE_ERR_INVALID_ARG


WRONG = [
    ("codes", (E, O, I // 2), U8), ("codes", (E, O, I // 32, 16), U8), ("codes", (E, 16, I // 32, O), U8), ("codes", (E, I // 2, O), U8), ("codes", (E, 16, O, I // 32), U8),
    ("scales", (E, O, I // G), BF16), ("scales", (I // G, E, O), BF16), ("scales", (O, E, I // G), BF16), ("scales", (E * O, I // G), BF16),
    ("zeros", (E, O, I // G), U8), ("zeros", (I // G, E, O), U8), ("zeros", (E * O, I // G), U8)]


@pytest.mark.parametrize("name,shape,dtype", WRONG)
def test_another_order_is_refused(name, shape, dtype):
    _refuses(_layer(**{name: torch.zeros(shape, dtype=dtype)}), "codes|scales|zeros")


@pytest.mark.parametrize("name,shape,dtype", [("codes", (O, I // 2), U8), ("codes", (O, I // 32, 16), U8), ("scales", (O, I // G), BF16), ("zeros", (O, I // G), U8)])
def test_another_order_of_a_plain_layer_is_refused(name, shape, dtype):
    _refuses(_layer(1, **{name: torch.zeros(shape, dtype=dtype)}), "codes|scales|zeros")


@pytest.mark.parametrize("E", [1, 3])
@pytest.mark.parametrize("join", ["as documented", "flat", "first two", "last two", "without experts"])
def test_joined_dimensions_are_the_same_layer(E, join):
    if join == "without experts" and E > 1:
        pytest.skip("several experts")
    change = {"as documented": lambda t: t, "flat": lambda t: t.reshape(-1), "first two": lambda t: t.flatten(0, 1), "last two": lambda t: t.flatten(-2, -1),
              "without experts": lambda t: t[0]}[join]
    d, codes, scales, zeros = _layer(E)
    _refuses((d, change(codes), change(scales), change(zeros)), "current device")


def test_biases():
    _refuses(_layer(), "bias", bias=torch.zeros((O, E), dtype=BF16))
    _refuses(_layer(), "bias", bias=torch.zeros(O, dtype=BF16))
    for shape in ((E, O), (E * O,), (E, 1, O)):
        _refuses(_layer(), "current device", bias=torch.zeros(shape, dtype=BF16))
    for shape in ((O,), (1, O), (O, 1)):
        _refuses(_layer(1), "current device", bias=torch.zeros(shape, dtype=BF16))


def test_slots():
    choice, offsets, rows = torch.zeros((6, 2), dtype=I32), torch.zeros(5, dtype=I32), torch.zeros(12, dtype=I32)
    for shape, what in (((2, 6), "sizes"), ((3, 4), "sizes"), ((6, 2), "current device"), ((12,), "current device")):
        with pytest.raises(B.PipeError, match=what):
            B.pipe_expert_rows(choice, 4, offsets, rows, torch.zeros(shape, dtype=I32))
    for shape in ((0, 2), (0,)):
        with pytest.raises(B.PipeError, match="current device"):
            B.pipe_expert_rows(torch.zeros((0, 2), dtype=I32), 4, offsets, torch.zeros(0, dtype=I32), torch.zeros(shape, dtype=I32))


@pytest.mark.parametrize("shape", [(), (O,), (1, 5, O)])
def test_rows_that_are_no_matrix_are_an_argument_error(shape):
    good_x, good_y = torch.zeros((5, I), dtype=BF16), torch.zeros((5, O), dtype=BF16)
    bad = torch.zeros(shape, dtype=BF16)
    for x, y in ((bad, good_y), (good_x, bad)):
        for call in (lambda: B.pipe_group_linear(*_layer(1), x, y), lambda: B.pipe_expert_linear(*_layer(), x, torch.zeros(E + 1, dtype=I32), y)):
            with pytest.raises(B.PipeError, match="matrices"):
                call()
    for y, out in ((bad, good_y), (good_y, bad)):
        with pytest.raises(B.PipeError, match="matrices"):
            B.pipe_expert_combine(y, torch.zeros((5, 2), dtype=I32), torch.zeros((5, 2)), out)
