"""The example that runs the attention operators together."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from tests.attention_ref import Attention, near  # noqa: E402


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_cache.py")
    spec = importlib.util.spec_from_file_location("attention_cache", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_last_decoded_token(example):
    q, k, v, args, out, weights = example.decode()
    ref = Attention(q, k, v, **args)
    near(out, ref.out, ref.out_err, "out")
    # 300 prompt tokens and 60 more in 320 slots: cut once to 256 when full, 20 tokens in
    assert int(args["lr"][0, 0, 1]) + 1 == 256 + 40
    # the newest row got weight from one token alone
    last = weights[:, :, 295].double()
    near(last, ref.weights[:, :, 295], ref.weights_err[:, :, 295] + 1e-6 * ref.weights[:, :, 295], "weights")


def test_shared_and_train(example):
    out, lse = example.shared()
    assert out.shape == (6, 8, 64) and bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    assert all(bool(torch.isfinite(t).all()) and bool(t.any()) for t in example.train())
