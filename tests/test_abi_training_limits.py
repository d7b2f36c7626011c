"""Limits that the init calls of the token tables and of AdamW state (no GPU needed)."""
import pytest

from test_abi_training_ops import _adamw, _embedding, lib  # noqa: F401


@pytest.mark.parametrize("eps", [1e-39, 1.1754942e-38, 1e-45])
def test_eps_of_8_bit_moments_is_no_subnormal_number(lib, eps):  # noqa: F811
    assert _adamw(lib, eps=eps, bits=8) == -1
    assert _adamw(lib, eps=2.0 ** -126, bits=8) != -1            # (there may be no device to go on with)
    assert _adamw(lib, eps=eps, bits=32) != -1


@pytest.mark.parametrize("value", [1e39, 3.41e38, 1.7e308])
@pytest.mark.parametrize("name", ["weight_decay", "lr_scale"])
def test_factors_are_finite_as_float32(lib, name, value):  # noqa: F811
    assert _adamw(lib, tensor={name: value}) == -1
    assert _adamw(lib, tensor={name: 3.4e38}) != -1              # (there may be no device to go on with)


@pytest.mark.parametrize("dim", [(1 << 22) + 1, 1 << 23])
def test_rows_end_at_their_limit(lib, dim):  # noqa: F811
    assert _embedding(lib, dim=dim) == -7
    assert _embedding(lib, dim=1 << 22, max_tokens=0) != -7
