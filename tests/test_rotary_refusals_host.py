"""Arguments of the stretched rotations that have no meaning are refused as such."""
import pytest

from paper_2510_26577_b200.rotary import inverse_frequencies


@pytest.mark.parametrize("kw", [dict(base=1.0), dict(beta_fast=0.0), dict(beta_slow=0.0), dict(beta_fast=-1.0), dict(beta_slow=float("nan"))])
def test_yarn(kw):
    with pytest.raises(ValueError):
        inverse_frequencies(64, **{"base": 10000.0, **kw}, scaling="yarn", factor=4.0, context=4096, device="cpu")
    inverse_frequencies(64, 10000.0, scaling="yarn", factor=4.0, context=4096, device="cpu")
