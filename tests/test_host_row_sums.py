"""The arithmetic of a row's softmax sums (csrc/row_sums.h) over the range of logits and temperatures that the calls accept, on the
CPU."""
from test_host_tile_grid import run_driver


def test_sums_over_the_range_of_logits_and_temperatures(tmp_path):
    assert int(run_driver("row_sums_driver", tmp_path).split()[0]) > 100_000


def test_gradients_over_the_range_of_logits_and_temperatures(tmp_path):
    assert int(run_driver("row_grad_driver", tmp_path).split()[0]) > 100_000
