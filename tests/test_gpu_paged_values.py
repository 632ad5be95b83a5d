"""Attention over a paged latent cache where its arithmetic can go wrong: what a bfloat16 layer rounds, probabilities far below the
largest, numbers that are none, lengths beyond the bound, page entries out of range."""

import numpy as np
import pytest
import torch

import paper_2407_21118_amd as P
from oracle import palu_oracle as O
from workloads import synth

pytestmark = pytest.mark.gpu

from gpu_util import make_desc, say, torch_dtype  # noqa: E402
from test_gpu_paged import LAYERS, Pool, hold  # noqa: E402


@pytest.mark.parametrize("name,prefix", [("4x256", 0), ("1x64", 0), ("gqa4", 0), ("8x512", 0), ("4x128-384", 0),
                                         ("4x256", 200), ("1x64", 200), ("gqa70", 200), ("3x384-64", 200)])
def test_a_bfloat16_layer_rounds_its_output_alone(name, prefix):
    """The output is the exact one rounded once: off by half a step of its own binade, and by what the sums before it are off.
    Keys and queries are pairs of float16 numbers (2^-21 of a product), composed angles right to 1e-6, so a logit of
    sum(|q k|) / sqrt(128) < 24 is right to 24 * 2.2e-6 = 2^-14.2 and so are probabilities, relative; these and the merged latents
    are pairs of bfloat16 numbers (2^-16 each).  Together 2^-13 of the row's largest output.  A key or a query rounded to
    11 bits moves a logit by up to 2^-11 of the same sum, 2^-9 of the output where few rows carry it."""
    lens = [333, 200, 257] if not prefix else [201 + 7 * i for i in range(21)]
    pool = Pool(LAYERS[name](), "bf16", lens, 16, seed=30, prefix=prefix)
    pool.put(0, 0)
    got = pool.call(pool.device()).double().cpu().numpy()
    ref = pool.reference()
    half = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(ref), 2.0 ** -100))) - 8)
    room = half + 2.0 ** -13 * np.abs(ref).max(-1, keepdims=True)
    off = np.abs(got - ref)
    beyond = np.maximum(off - half, 0) / np.abs(ref).max(-1, keepdims=True)
    say(f"[paged] {name}, prefix {prefix}: beyond half a step by at most {beyond.max():.2e} of the row's largest")
    assert (off <= room).all(), beyond.max()
