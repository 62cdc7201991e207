"""What the co-inference command refuses, before anything is built or timed (so this runs without a GPU)."""

import pytest

from paper_2504_14611_amd import coinference as co


@pytest.mark.parametrize("argv", [["--cache-bits", "8"], ["--cache-bits", "8", "--page", "0"], ["--page", "-16"], ["--page", "65537"]])
def test_refused_options(argv, capsys):
    pytest.importorskip("torch")
    with pytest.raises(SystemExit) as end:
        co.main(argv)
    assert end.value.code == 2 and "--page" in capsys.readouterr().err


@pytest.mark.parametrize("page", [-16, 65537])
def test_refused_pages(page):
    pytest.importorskip("torch")
    shape = co.Shape(blocks=1, width=64, heads=2, kv_heads=1, inner=64, rank=4)
    with pytest.raises((ValueError, co.jdob.JdobError)):
        co.Edge(shape, co.make_chain(shape, 1, device="cpu"), [0], 0, 40, device="cpu", page=page)
