"""What the attentions' softmax and weighted sums lose, on inputs that show it (edge_precision_model)."""

import pytest
import torch

from paper_2504_14611_amd import edge
from tests import edge_precision_model as model

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def paged(scores, v, base, new, page, dtype, bits8, part, v_scale=None, kv_heads=2, group=2, label=None,
          reach=128):
    s = model.paged(scores, v, base, new, page, kv_heads, group, dtype, bits8, v_scale)
    got = edge.attend_paged(s["q"], s["cache"], s["table"], s["row_start"], s["key_count"], scale=1.0, max_queries=new,
                            max_keys=len(scores))
    values = v if v_scale is None else v.double() * v_scale.double()[:, None]
    over = model.over(got, scores, values, new, dtype, part, reach)
    assert over <= 0, (label, over)


BASES = [0, 1 << 12, 1 << 20, 1 << 23, -(1 << 23)]


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("page", [16, 20, 7])
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_scores_far_from_zero_over_pages(dim, page, dtype, bits8):
    """Waves and workgroups whose maxima differ, scores far from zero: weights are those of the differences."""
    for base in BASES:
        for keys, new, group in ((64, 1, 2), (600, 3, 2), (5000, 1, 4), (3000, 5, 8)):
            for seed in (0, 1):
                scores, v = model.far_scores(keys, seed, "cuda", dim)
                paged(scores, v, base, new, page, dtype, bits8, 2.0 ** -16, group=group, label=(base, keys, new, seed))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_scores_far_from_zero(dim, dtype):
    """Packed keys: few rows, whose keys are split over waves and workgroups, and many."""
    for base in BASES:
        for what, keys, new in ((model.far_scores, 64, 1), (model.far_scores, 3000, 3), (model.rising_scores, 600, 2),
                                (model.rising_scores, 600, 200), (model.far_scores, 700, 200)):
            for seed in (0, 1):
                scores, v = what(keys, seed, "cuda", dim)
                q, k, v16, *where = model.packed(scores, v, base, new, 2, 2, dtype)
                got = edge.attend(q, k, v16, *where, scale=1.0, max_queries=new, max_keys=keys)
                over = model.over(got, scores, v, new, dtype, model.HALF[dtype])
                assert over <= 0, (base, what, keys, new, seed, over)


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("page", [16, 20, 7])
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_small_weights(dim, page, dtype, bits8):
    """Weights of e^-5 to e^-60 beside one of 1 whose value is zero, in the same tile, wave and workgroup and in others."""
    for keys, new, group in ((500, 1, 2), (5000, 1, 4), (3000, 5, 8)):
        for above in (5, 15, 17, 18, 25, 60):
            scores, v, v_scale = model.small_weights(keys, above, "cuda", dim)
            if bits8:
                paged(scores, v, 0, new, page, dtype, True, 2.0 ** -16, v_scale, group=group, label=(keys, new, above))
            else:
                paged(scores, v * v_scale[:, None], 0, new, page, dtype, False, 2.0 ** -16, group=group, label=(keys, new, above))


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("page", [16, 20, 7])
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_huge_values(dim, page, bits8):
    """Sums that pass binary32 before they are divided, in one wave and where waves and workgroups are joined."""
    for keys, new, group in ((1, 1, 2), (200, 1, 2), (5000, 1, 4), (3000, 5, 8), (70000, 1, 2)):
        scores, v, v_scale = model.huge_values(keys, keys, "cuda", dim)
        if bits8:
            paged(scores, v, 0, new, page, BF16, True, 2.0 ** -16, v_scale, group=group, label=(keys, new))
        else:
            paged(scores, v * v_scale[:, None], 0, new, page, BF16, False, 2.0 ** -16, group=group, label=(keys, new))


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("page", [16, 20, 7])
@pytest.mark.parametrize("dim", [64, 96, 128])
def test_weights_keep_16_bits(dim, page, dtype, bits8):
    """Sums of terms that cancel: a weight of one part, 8 or 11 bits, would show."""
    for keys in (2, 5, 20, 60, 300, 2000):
        for seed in range(2):
            scores, v, v_scale = model.cancelling_values(keys, seed, dtype, bits8, "cuda", dim)
            for group in (2, 8):
                paged(scores, v, 0, 1, page, dtype, bits8, 2.0 ** -16, v_scale if bits8 else None, group=group, reach=9,
                      label=(keys, seed))


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("scale", [1e30, 2.9e38])
def test_scales_near_the_end_of_binary32(scale, bits8):
    """Every row is the value of the key with its largest score."""
    scores = (torch.arange(100, device="cuda") * 37) % 101
    v = torch.randint(-100, 100, (100, 64), generator=torch.Generator().manual_seed(1)).float().cuda()
    want = torch.stack([v[scores[:97 + i + 1].argmax()] for i in range(3)])[:, None].expand(3, 4, 64)
    s = model.paged(scores, v, 0, 3, 16, 2, 2, BF16, bits8)
    got = edge.attend_paged(s["q"], s["cache"], s["table"], s["row_start"], s["key_count"], scale=scale, max_queries=3, max_keys=100)
    assert torch.equal(got.float(), want)
    q, k, v16, *where = model.packed(scores, v, 0, 3, 2, 2, BF16)
    for most in (3, 200):
        assert torch.equal(edge.attend(q, k, v16, *where, scale=scale, max_queries=most, max_keys=100).float(), want), most
