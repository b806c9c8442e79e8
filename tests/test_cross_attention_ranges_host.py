"""Cross attention: configurations whose operands would span more elements than the kernels address are refused, also where the product of
length and stride passes 63 bits.  Needs no GPU."""
import ctypes

import pytest

from paper_2006_16668_b200 import binding as B
from paper_2006_16668_b200.build import build_library

P = [0x10000 * (i + 1) for i in range(12)]


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()


def _sizes(q_len=1, k_len=1, q_stride=64, k_stride=64, v_stride=64):
    c = B.gshard_attention_config(1, q_len, k_len, 1, 1, 64, B.GSHARD_BF16, 0.125, q_stride, k_stride, v_stride)
    lib, p = B.load(), ctypes.byref(c)
    sizes = {lib.gshard_cross_attention_workspace_bytes(p, back) > 0 for back in (0, 1)}
    codes = {lib.gshard_cross_attention_forward(p, *P[:6], P[6], 0, None), lib.gshard_cross_attention_backward(p, *P[:10], P[10], 0, None)}
    return sizes, codes


@pytest.mark.parametrize("length", [1 << 30, (1 << 30) - 1, 1 << 28, 3 << 27, 1 << 20])
@pytest.mark.parametrize("stride", [(1 << 36) - 8, 1 << 35, 1 << 34, 3 << 33, 1 << 33])
@pytest.mark.parametrize("which", ["q", "k", "v"])
def test_spans_of_more_than_38_bits(which, length, stride):
    assert length * stride >= 1 << 38
    lengths = {"q_len": length} if which == "q" else {"k_len": length}
    assert _sizes(**lengths, **{which + "_stride": stride}) == ({False}, {B.GSHARD_ERR_UNSUPPORTED_SHAPE})


@pytest.mark.parametrize("length,stride", [(1, (1 << 36) - 8), (4, (1 << 36) - 8), ((1 << 20) - 1, 1 << 18), (1 << 18, (1 << 20) - 8), (0, (1 << 36) - 8)])
@pytest.mark.parametrize("which", ["q", "k", "v"])
def test_spans_below_it(which, length, stride):
    assert length * stride < 1 << 38
    lengths = {"q_len": length} if which == "q" else {"k_len": length}
    sizes, codes = _sizes(**lengths, **{which + "_stride": stride})
    assert sizes == {True} and codes <= {B.GSHARD_OK, B.GSHARD_ERR_WORKSPACE_TOO_SMALL}
