"""The oracle's attention against closed forms and loops, and the argument checks of the attention calls that need no GPU."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import cake_oracle as O
from paper_2503_12491_b200 import binding


def test_uniform_keys_average_what_is_visible():
    q, k = np.ones((2, 4, 8)), np.zeros((1, 4, 8))
    v = np.arange(32.0).reshape(1, 4, 8)
    out, lse, _ = O.prompt_attention(q, k, v)
    for i in range(4):
        assert np.allclose(out[:, i], v[0, :i + 1].mean(0)) and np.allclose(lse[:, i], np.log(i + 1))


def test_prompt_attention_agrees_with_softmax_rows_and_cumulative_attention():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(4, 19, 8)), rng.normal(size=(2, 19, 8)), rng.normal(size=(2, 19, 8))
    out, lse, _ = O.prompt_attention(q, k, v)
    received = np.zeros((2, 19))
    for h in range(4):
        s = q[h] @ k[h // 2].T / np.sqrt(8.0)
        p = np.tril(np.exp(s - lse[h][:, None]))
        assert np.allclose(p.sum(1), 1.0) and np.allclose(p @ v[h // 2], out[h])
        received[h // 2] += p.sum(0) / 2
    assert np.allclose(received, O.cumulative_attention(q, k))


def test_rows_that_see_nothing_and_what_lies_behind():
    k, v = np.ones((3, 4)), np.ones((3, 4))
    k[2], v[2] = np.nan, np.inf
    out, lse, _ = O.attend(np.ones((2, 4)), k, v, np.array([[False] * 3, [True, True, False]]))
    assert np.array_equal(out[0], np.zeros(4)) and lse[0] == -np.inf
    assert np.allclose(out[1], 1.0) and np.isfinite(lse[1])


@pytest.mark.parametrize("group", [32, 64])
def test_dequantised_rows_lie_within_half_a_step(group):
    x = np.random.default_rng(1).normal(size=(75, 64)).astype(np.float32)
    q, s, z = O.quantize_keys_per_channel(x, group)
    assert np.array_equal(O.unpack_nibbles(O.pack_nibbles(q)), q)
    step = np.repeat(s, group, axis=0)[:75]
    assert (np.abs(O.dequantize_keys(q, s, z, group) - x) <= 0.5001 * step + 1e-6).all()
    q, s, z = O.quantize_values_per_token(x, group)
    assert (np.abs(O.dequantize_values(q, s, z, group) - x) <= 0.5001 * np.repeat(s, group, axis=1) + 1e-6).all()


def test_null_arguments_are_refused():
    lib = binding.load_library()
    n, i = None, ctypes.c_int64(0)
    assert lib.cake_attend_prompt(n, n, i, i, n, n, n, i, i, n, n, n) == binding.CAKE_ERR_ARG
    assert lib.cake_accumulate_attention(n, n, i, i, n, n, n, n) == binding.CAKE_ERR_ARG
    assert lib.cake_attend_workspace_bytes(n, 1) == binding.CAKE_ERR_ARG
    assert lib.cake_attend_cache(n, 1, 0, n, n, n, n, n, n, n, i, n, n, n, i, n) == binding.CAKE_ERR_ARG
    assert lib.cake_attend_int4(n, 1, 0, n, n, n, n, n, n, n, 32, n, n, n, n, n, i, n, n, n, i, n) == binding.CAKE_ERR_ARG


def test_the_native_marshalling_refuses_what_is_no_cuda_tensor():
    binding.load_library()
    q, k = torch.zeros(2, 4, 64), torch.zeros(2, 4, 64)
    with pytest.raises(ValueError, match="CUDA tensors only"):
        binding._fast.attend_prompt(0, True, 1, 4, 2, 2, 64, 1, q, k, k, None, None, None)
    with pytest.raises(ValueError, match="expected a torch.Tensor"):
        binding._fast.accumulate_attention(0, True, 4, 2, 2, 64, 1, k, k, None)
    with pytest.raises(ValueError, match="CUDA tensors only"):
        binding._fast.attend_cache(0, True, 0, 1, 2, 2, 64, q, k, None, None, None, None, None, k, k)
    with pytest.raises(TypeError, match="arguments"):
        binding._fast.attend_int4(0, True, 0)
