"""Device code that the host compiler runs (tests/native): index arithmetic, and a block thread by thread in orders that a GPU
seldom takes."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


def run_native(name, tmp_path, *flags):
    exe = os.path.join(tmp_path, name)
    subprocess.run(["g++", "-O1", "-g", "-std=c++17", *flags, "-o", exe, os.path.join(HERE, "native", name + ".cpp")], check=True, timeout=300)
    done = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert done.returncode == 0, done.stdout


def test_search_for_the_largest_elements_in_any_order_of_warps(tmp_path):
    run_native("top_search", tmp_path)


def test_granules_that_are_read_lie_inside(tmp_path):
    run_native("ranges", tmp_path)
