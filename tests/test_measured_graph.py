"""CPU check of the measured iteration's graph: every op depends on what it reads and on nothing else."""

from paper_1803_03288_amd import measured


def test_edges_are_what_the_ops_read():
    g = measured.iteration_graph(2, 64, 256)
    after = dict(g.ops)
    for i in range(2):
        x = ["forward.add0"] if i else []
        assert after[f"forward.norm{i}"] == [f"norm{i}"] + x
        assert after[f"forward.linear1.{i}"] == [f"forward.norm{i}", f"w1.{i}", f"b1.{i}"]
        assert after[f"forward.relu{i}"] == [f"forward.linear1.{i}"]
        assert after[f"forward.linear2.{i}"] == [f"forward.relu{i}", f"w2.{i}", f"b2.{i}"]
        assert after[f"forward.add{i}"] == [f"forward.linear2.{i}"] + x
        dx = "loss" if i else "backward.add1"
        assert after[f"backward.linear2.{i}"] == [dx, f"forward.relu{i}", f"w2.{i}"]
        assert after[f"backward.relu{i}"] == [f"backward.linear2.{i}", f"forward.relu{i}"]          # (its mask is an output of the relu)
        assert after[f"backward.linear1.{i}"] == [f"backward.relu{i}", f"forward.norm{i}", f"w1.{i}"]
        assert after[f"backward.norm{i}"] == [f"backward.linear1.{i}", f"forward.norm{i}", f"norm{i}"]
        assert after[f"backward.add{i}"] == [f"backward.norm{i}", dx]
    assert after["loss"] == ["forward.add1"]
