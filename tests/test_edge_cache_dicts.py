"""Caches that lack a tensor are refused like others that do not fit (so this runs without a GPU)."""

import pytest
import torch

from paper_2504_14611_amd import edge, jdob


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("name", ["k", "v"])
@pytest.mark.parametrize("how", [lambda c, n: {**c, n: None}, lambda c, n: {m: t for m, t in c.items() if m != n}])
def test_a_cache_without(how, name, bits8):
    cache = how(edge.make_cache(4, 16, 2, 64, bits8=bits8, device="cpu"), name)
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    i32 = torch.int32
    where = torch.zeros(1, 4, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(1, dtype=i32)
    for call in (lambda: edge.cache_write(x, x, cache, *where), lambda: edge.cache_read(cache, *where, rows=3),
                 lambda: edge.cache_read(cache, *where, into={"k": x, "v": x}), lambda: edge.attend_paged(x, cache, *where)):
        with pytest.raises(jdob.JdobError):
            call()
