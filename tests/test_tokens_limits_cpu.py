"""The token calls (include/az_tokens.h) where they may not work: refusals at their limits, before any CUDA call, and their compiled
binding missing."""
import os
import subprocess
import sys

import pytest

import paper_2609_37447_b200 as az

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_the_status_self_test_knows_two_parts():
    assert az._lib.az_selftest_tokens_timeout(2, None) == az.AZ_ERR_BAD_ARG
    assert az._lib.az_selftest_tokens_timeout(-1, None) == az.AZ_ERR_BAD_ARG


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantise_refuses_more_blocks_than_a_grid_holds(block_rows):
    most, address = 2 ** 31 - 1, 1 << 20
    assert az._lib.az_quantise_blocks(address, az.AZ_TYPE_BF16, most, most, most, block_rows, address, most, address, 1 << 24,
                                      None) == az.AZ_ERR_UNSUPPORTED


def test_product_refuses_more_tiles_than_it_counts():
    """Before any CUDA call: here there is no device to ask."""
    address, side, k = 1 << 20, 1 << 24, 16
    assert az._lib.az_block_matmul(address, k, address, 1, address, k, address, 1, None, side, side, k, address, az.AZ_TYPE_F32, side,
                                   None) == az.AZ_ERR_UNSUPPORTED


def test_the_package_without_the_binding_of_the_token_calls():
    """The engine's calls work; the token calls say what is missing, each time."""
    code = """
import sys
sys.modules["paper_2609_37447_b200._tokens"] = None
import torch, paper_2609_37447_b200 as az
assert az.az_strerror(0) == "ok" and az.az_policy_size(az.make_arch(19, 20, 128, 1, 1, 1, 1024)) == 1858
x = torch.zeros(2, 128)
for call in (lambda: az.az_adjust_logits(x, x), lambda: az.az_token_probs(x, x), lambda: az.az_adjust_logits(x, x)):
    try:
        call()
    except ImportError as e:
        assert "_tokens.so" in str(e) and "build" in str(e)
    else:
        raise AssertionError
del sys.modules["paper_2609_37447_b200._tokens"]
try:
    az.az_adjust_logits(x, x)
except TypeError as e:
    assert "CUDA tensor" in str(e)
else:
    raise AssertionError
"""
    subprocess.run([sys.executable, "-c", code], check=True, cwd=ROOT, timeout=300)


def test_a_binding_that_does_not_compile_leaves_the_library(monkeypatch, tmp_path):
    import __graft_entry__
    build = __graft_entry__.load_build_module()
    lib = build.build()
    for name in ("BINDING", "BINDING_STAMP"):
        monkeypatch.setattr(build, name, str(tmp_path / name))
    monkeypatch.setattr(build, "_binding_command", lambda: ["false"])
    with pytest.raises(RuntimeError, match="is built, the binding"):
        build.build()
    assert os.path.exists(lib) and not os.path.exists(tmp_path / "BINDING_STAMP")
