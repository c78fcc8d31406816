"""The example resumes from its checkpoints alone."""
import importlib.util
import os

import pytest
import torch

import paper_2010_08679_amd as P

pytestmark = pytest.mark.gpu


def test_the_example_resumes_from_nothing_but_checkpoints():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "train_and_decode.py")
    spec = importlib.util.spec_from_file_location("train_and_decode", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.main()
    for trained, resumed in zip(r["trained_matrices"], r["resumed_matrices"]):
        # other memory, and each row within half a step of 8 bits over its range
        assert trained.data_ptr() != resumed.data_ptr() and not torch.equal(trained, resumed)
        step = (trained.amax(dim=1) - trained.amin(dim=1)) / 255
        assert bool(((trained - resumed).abs() <= step[:, None] * 0.51 + 1e-6).all())
    ctx = P.cnr_create(0)
    assert example.decode(ctx, *r["resumed_matrices"], r["prompts"], 12, forbidden=[38]) == r["resumed"]
    P.cnr_destroy(ctx)
