"""The graph of the measured iteration with weights in 8-bit floats by blocks (``paper_1803_03288_amd.measured``)."""

import pytest

from paper_1803_03288_amd import measured


def test_graph_of_the_blocks():
    """The ops and their edges are those of the other iteration; what is sent is a byte per weight and one per block."""
    for width, hidden, blocks in ((64, 256, 2), (129, 130, 4), (1024, 4096, 256)):
        rows, by_block = measured.iteration_graph(3, width, hidden), measured.iteration_graph(3, width, hidden, True)
        assert by_block.ops == rows.ops
        for a, b in zip(rows.recvs, by_block.recvs):
            assert a[0] == b[0] and a[2] == b[2]
            assert b[1] == (width * hidden + blocks if a[0].startswith("w") else a[1])
    g = measured.iteration_graph(1, 64, 256, True)
    assert g.recvs[1] == ("w1.0", 64 * 256 + 2, 4 * 64 * 256) and len(g.csr()[1]) == g.csr()[0] + 1


@pytest.mark.parametrize("argv", [["--update", "16"], ["--blocks", "1"]])
def test_unknown_options(argv):
    with pytest.raises(SystemExit):
        measured.main(argv)
