"""The order in which an output layer's products walk over their tiles, run by the host compiler (tests/native/tiles.cpp)."""
from test_emulated_blocks import run_native


def test_every_tile_comes_once_and_divisions_are_exact(tmp_path):
    run_native("tiles", tmp_path)
