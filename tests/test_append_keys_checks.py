"""The checks of appended keys fail for what a kernel with a mistake would leave: on the host, the mistake planted in the reference."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import cache_util as U
from oracle import cache as R
from test_gpu_append_keys import check_bf16_keys, check_quant_keys

KINDS = ["none", "position", "page", "head", "slot"]


def case(kind):
    c = U.batch(133, ctx=[30, 10], n=[9, 12], heads=(2, 2), D=64)
    wrong = dict(c)
    if kind == "position":
        wrong["positions"] = np.concatenate([np.arange(9) + 31, np.arange(12) + 11]).astype(np.int32)
    if kind == "page":
        wrong["table"] = c["table"].copy()
        wrong["table"][0, 2] = next(p for p in range(c["held"]) if p not in c["table"])
    if kind == "head":
        wrong["k"] = c["k"][:, ::-1]
    if kind == "slot":
        wrong["k"] = np.roll(c["k"], 1, axis=0)
    return c, wrong


@pytest.mark.parametrize("kind", KINDS)
def test_bf16(kind):
    c, wrong = case(kind)
    before = U.bf16(c["rng"].standard_normal((c["held"], 2, 16, 64)))
    got = U.bf16(R.append(wrong, before, before)[1])
    if kind == "none":
        check_bf16_keys(c, before, got)
    else:
        with pytest.raises(AssertionError):
            check_bf16_keys(c, before, got)


@pytest.mark.parametrize("kind", KINDS)
def test_quant(kind):
    c, wrong = case(kind)
    before = U.quant_pools(c)
    got = R.append_quant(wrong, *before)[1]
    if kind == "none":
        check_quant_keys(c, before, got)
    else:
        with pytest.raises(AssertionError):
            check_quant_keys(c, before, got)
