"""The example that runs pages, adapters and attention together as a serving program does, against the same model in 64 bits."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_step.py")


@pytest.mark.parametrize("dtype,bound", [(torch.float32, 1e-4), (torch.bfloat16, 0.1)])
def test_steps_of_a_small_decoder(dtype, bound):
    """Bounds: two layers of a projection, LoRA, attention and a projection, each of which rounds its rows to the type.  f32: sums of 512 terms at 2^-24 each, through
    eight such stages, 8 * 512 * 2^-24 = 2.4e-4 at the very worst and its root in practice.  bf16: at 2^-8 a rounding, some 12 roundings in a chain, with gains of
    about one: 12 * 2^-8 = 0.05, twice that for the products of perturbed scores."""
    print(f"\n[case] serve_step {dtype}", flush=True)
    spec = importlib.util.spec_from_file_location("serve_step", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    worst = module.main(dtype)
    print(f"  off by {worst:.2e}", flush=True)
    assert worst <= bound
