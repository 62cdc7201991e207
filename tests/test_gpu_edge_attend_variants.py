"""Every kernel that jdob_edge_attend chooses from, against the definition in 64 bits: each head size's tiles, rows at
16 bytes and at any element, few rows (keys split or not) and many, values that some rows must not see."""

import pytest
import torch

from paper_2504_14611_amd import edge
from tests.test_gpu_edge_attend import BF16, F16, check, inputs

pytestmark = pytest.mark.gpu


def moved(t, shift):
    """The same values from `shift` elements behind an aligned address on."""
    flat = torch.empty(t.numel() + 8, dtype=t.dtype, device="cuda")
    view = flat[shift:shift + t.numel()].view(t.shape)
    return view.copy_(t)


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("dim", [8, 64, 72, 96, 104, 128])
@pytest.mark.parametrize("new,keys", [([1, 3], [200, 40]), ([2], [2500]), ([1, 1], [1500, 0]), ([150, 9], [170, 5]),
                                      ([70, 200], [60, 333])])
def test_attend_variants(new, keys, dim, dtype, shift):
    s = inputs(new, keys, 4, 2, dim, dtype, seed=dim + sum(keys))
    s.update({name: moved(s[name], shift) for name in "qkv"})
    clean = check(s, "clean")
    assert torch.equal(clean, edge.attend(**{**s, **{name: moved(s[name], 0) for name in "qkv"}}))
    # the last sequence's last value: its last row alone sees it
    at = int(s["key_start"][-1]) + keys[-1] - 1
    if keys[-1]:
        s["v"][at] = float("inf")
        got = edge.attend(**s)
        assert torch.equal(got[:-1], clean[:-1]) and not got[-1].isfinite().any()
