"""Rules that choose between forms of the few-bit products: the library's own host code, no GPU call."""
import shutil

import pytest

from test_host_logic import _run_host_program


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="no hipcc")
def test_forms_of_few_bit_products(tmp_path):
    _run_host_program("few_bits.hip", tmp_path, "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops")


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="no hipcc")
def test_limits_of_few_bit_products(tmp_path):
    _run_host_program("few_bits_limits.hip", tmp_path, "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops")


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="no hipcc")
def test_plans_of_weight_gradients(tmp_path):
    _run_host_program("few_bits_plans.hip", tmp_path, "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops")
