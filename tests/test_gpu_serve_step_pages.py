"""The example's steps with head norms and rotated keys, over pages of the rows' type and of 4-bit numbers, against the same model in 64 bits."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_step.py")


@pytest.mark.parametrize("keys", ["turned", "four"])
@pytest.mark.parametrize("dtype,bound", [(torch.float32, 1e-4), (torch.bfloat16, 0.1)])
def test_steps_of_a_small_decoder(keys, dtype, bound):
    """The bounds of the plain steps: sums of 512 terms at 2^-24 through eight stages, 2.4e-4 at the very worst and its root in practice; in bf16 some 12 roundings in a
    chain, 12 * 2^-8 = 0.05, twice that for the products of perturbed scores.  The norms and the rotation add one rounding to queries and keys; 4-bit pages add none, as
    the model in 64 bits reads what they hold (and the example checks that against its own keys and values)."""
    print(f"\n[case] serve_step {keys} {dtype}", flush=True)
    spec = importlib.util.spec_from_file_location("serve_step", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    worst = module.main(dtype, keys=keys)
    print(f"  off by {worst:.2e}", flush=True)
    assert worst <= bound
