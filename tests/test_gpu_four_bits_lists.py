"""Decode over rows held in 4 bits where a workgroup takes several KV heads together (batches of many
sequences, and lists longer than its room for relevance values, which is then emptied on the way).
tests/test_attention_split_four_cpu.py pins that these lists have that form."""
import pytest

from tests.test_attention_split_four_cpu import GPU_CASES
from tests.test_gpu_four_bits import _long_step, _run, _workload, gpu  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name,Hq,tau,relevance", [
    ("longer-rows64", 32, 6.3, "abs"), ("longer-rows64", 64, 6.3, "abs"), ("longer-rows128", 32, 8.0, "abs"),
    ("longer-rows128", 64, 8.0, "abs"), ("longer-rows256", 16, 12.7, "abs"), ("longer-softmax", 64, 2.6e-5, "softmax")])
def test_longer_lists(name, Hq, tau, relevance):
    n, hkv, dim, planes, hw, full = GPU_CASES[name]
    assert hw == 8 and full and planes == (1 if relevance == "abs" else Hq // hkv)
    _long_step([x - 1 for x in n], Hq, hkv, dim, tau, relevance)


@pytest.mark.parametrize("name,Hq", [("together-40", 32), ("together-40", 64), ("together-70", 8), ("together-70", 64),
                                     ("together-70-rows256", 16), ("together-70-rows256", 64), ("together-300", 32)])
def test_heads_together(name, Hq):
    n, hkv, dim, _, hw, _ = GPU_CASES[name]
    assert hw > 1
    _run(_workload(batch=len(n), prefill=[x - 1 for x in n], n_q_heads=Hq, n_kv_heads=hkv, head_dim=dim, steps=3,
                   f_hh=[0.3] * len(n)), with_logits=False)
