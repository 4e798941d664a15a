"""Where the lm_head operators' products read and write (csrc/head_tile.h), walked on the CPU."""
from test_host_tile_grid import run_driver


def test_every_access_stays_inside_its_array(tmp_path):
    assert int(run_driver("head_tile_driver", tmp_path).split()[0]) > 10_000_000
