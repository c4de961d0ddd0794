"""Arrays of the 8-bit integer layers are taken in the documented shape, dimensions joined or of one put in, alone."""
import pytest
import torch

from paper_2311_15806_b200 import binding as B


def _arrays(E, O, I, shape, N=6):
    codes = torch.zeros((*shape, I), dtype=torch.int8)
    return codes, torch.zeros((E, O)), torch.zeros((N, I), dtype=torch.int8), torch.zeros(N), torch.zeros((N, O), dtype=torch.bfloat16)


def _reason(call):
    with pytest.raises(B.PipeError) as e:   # (of CPU tensors: at the latest for their device)
        call()
    return str(e.value)


@pytest.mark.parametrize("E,O,shape,good", [(2, 3, (2, 3), True), (2, 3, (6,), True), (2, 3, (3, 2), False), (2, 3, (1, 6), True), (2, 3, (6, 1), True), (4, 4, (2, 8), False),
                                            (2, 3, (5,), False), (2, 3, (2, 4), False), (1, 6, (6,), True), (1, 6, (1, 6), True), (1, 6, (6, 1), True), (1, 6, (2, 3), False)])
def test_codes_of_another_order_are_refused(E, O, shape, good):
    codes, scales, xq, sx, y = _arrays(E, O, 32, shape)
    d = B.make_int8_desc(O, 32, experts=E)
    offsets = torch.zeros(E + 1, dtype=torch.int32)
    for call in [lambda: B.pipe_int8_expert_linear(d, codes, scales, xq, sx, offsets, y)] + ([lambda: B.pipe_int8_linear(d, codes, scales, xq, sx, y)] if E == 1 else []):
        assert ("current device" in _reason(call)) == good
