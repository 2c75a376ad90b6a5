"""Host: the closer bounds for attention over 8-bit pages hold for probabilities rounded to binary16
and fail for what a kernel could lose unseen under the wider ones."""
import pytest
import torch

from codes_ref import alternating_case, attend_codes64_close, make_code_case


def worst(got, want):
    out, _, ob, _ = want
    return float(((got - out).abs() / ob).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_closer_bounds_tell_binary16_probabilities_from_bf16(dtype):
    lens, window = [(40, 60), (3, 3)], 2
    q, keys, values, _, _, _ = alternating_case(lens, 2, 64, dtype, 16)
    run = lambda f=None: attend_codes64_close(q, keys, values, lens, 1, window, 0, round_p=f)
    want = run()
    assert worst(run(lambda w: (w * 2 ** 15).half().double() / 2 ** 15)[0].to(dtype).double(), want) <= 1
    assert worst(run(lambda w: w.bfloat16().double())[0].to(dtype).double(), want) > 1


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_closer_bounds_tell_where_probabilities_end(dtype):
    """One token draws most of the weight and has no Value: the others, 2^-23 of it, are the output."""
    lens = [(2, 400)]
    q, keys, values, _, _, _ = make_code_case(85, lens, 1, 1, 64, dtype, 16)
    q = torch.zeros_like(q)
    q[..., 5] = 1.0
    keys[0] = keys[0] * 0.01
    keys[0][0, 0, 5] = 16.0
    values[0] = values[0].abs() + 0.5
    values[0][0] = 0
    run = lambda f=None: attend_codes64_close(q, keys, values, lens, 1, 0, 0, scale=1.0, round_p=f)
    want = run()
    assert worst(run(lambda w: (w * 2 ** 15).half().double() / 2 ** 15)[0].to(dtype).double(), want) <= 1
    assert worst(run(lambda w: w.half().double())[0].to(dtype).double(), want) > 1     # 1 at the maximum: 2^-24 at the end
