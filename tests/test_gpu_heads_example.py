"""The example that trains, certifies and serves several tenants' heads."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_tenant_heads_example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import __graft_entry__
    __graft_entry__.build()
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "tenant_heads.py")
    spec = importlib.util.spec_from_file_location("tenant_heads", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    r = example.run()
    # Before training a tenant's moved classes (8 of 20) are all answered by the shared head, wrongly.
    assert 0.5 < r["accuracy_before"] < 0.7
    assert r["accuracy_after"] > 0.95
    assert r["loss"][-1] < 0.5 * r["loss"][0]
    assert r["answered"]
    assert r["hit_rate"] > 0.1
    # Certified hits: the tenant's own head gives the same label.
    assert r["hits_agree"] == 1.0
