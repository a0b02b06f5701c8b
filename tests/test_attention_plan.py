"""The attention plan (host-only C++) under the address and undefined-behaviour sanitizers: no GPU, no HIP."""
import os

from tests.test_sanitizers import HERE, _build_and_run


def test_attention_plan_under_sanitizers(tmp_path):
    _build_and_run(tmp_path, "g++", ["-std=c++17", os.path.join(HERE, "sanitize", "attention_plan_driver.cpp")], [])


def test_attention_plan_of_the_largest_windows_under_sanitizers(tmp_path):
    _build_and_run(tmp_path, "g++", ["-std=c++17", os.path.join(HERE, "sanitize", "attention_plan_window_driver.cpp")], [])
