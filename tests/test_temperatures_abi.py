"""Temperatures that the operators on logits refuse and accept, through the C ABI
on the CPU.  A call with an accepted temperature fails a later check (a misaligned
pointer), so nothing reaches a GPU."""
import math

import pytest

from test_ops_abi import ALIGN, BWD, FWD, SCORE, SHAPE, STEP, addr, call, lib  # noqa: F401


def test_token_logprobs_takes_normal_numbers(lib):
    # 1/T and log2(e)/T have to be finite, or a row's maximum gives 0 x inf
    for T in (1e-45, 1e-40, 2.0 ** -127, 1.17e-38, 0.0, math.inf):
        assert call(lib.lora_token_logprobs, SCORE, T=T) == SHAPE, T
    for T in (2.0 ** -126, 1e-30, 1e-6, 1.0, 1e30, 3.4e38):
        assert call(lib.lora_token_logprobs, SCORE, T=T, entropy=addr(3, 2)) == ALIGN, T


@pytest.mark.parametrize("name,base", [("lora_distill_fwd", FWD), ("lora_distill_bwd", BWD), ("lora_distill_step", STEP)])
def test_distillation_takes_temperatures_with_a_square(lib, name, base):
    fn = getattr(lib, name)
    for T in (1e-45, 2.0 ** -127, 1e-30, 2.0 ** -64, 2.0 ** 64, 1e30, 3.4e38, math.inf):
        assert call(fn, base, T=T) == SHAPE, T
    for T in (2.0 ** -63, 1e-10, 1.0, 1e10, 2.0 ** 63):
        assert call(fn, base, T=T, z=addr(0, 1)) == ALIGN, T
