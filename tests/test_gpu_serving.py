"""GPU: the serving path as a whole (paper_2310_07240_amd/serving.py) on a small cache: decode,
store, a question with weights, tokens, page selection, eviction, and back to the codec."""
import pytest

from paper_2310_07240_amd import workloads as W
from gpu_helpers import say, torch_cuda

pytestmark = pytest.mark.gpu


def test_serving_path():
    torch_cuda()
    from paper_2310_07240_amd import serving
    w = W.small(name="serving", n_layers=3, n_tokens=300, n_channels=256, chunk_len=128)
    r = serving.run(w, kv_heads=4, q_heads=8, question=70, tokens=3, keep=0.5, picks=4)
    say(r)
    assert r["sequences"] == w.n_ctx * 3 and r["tokens"] == 373 and r["kept"] == 186
    # a code is off by at most half a step, 1 / 254 of its page's largest value: the outputs, whose
    # weights shift with the keys, stay within a few percent of the fp16 cache's
    assert r["rel_error_8bit"] < 0.05
    assert 0 < r["kept_of_context"] <= 1
    assert r["bytes"]["pages"] < 0.65 * r["bytes"]["fp16"]
    assert set(r["ms"]) == {"decode", "store", "question", "token", "select", "sparse", "evict",
                            "load"}
