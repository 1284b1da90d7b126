"""GPU: requests that answer over contexts (paper_2310_07240_amd/serving.py, answer): pages reserved,
shared and copied, drafts attended over, verified and cut back, pages given back and moved."""
import json

import pytest

from paper_2310_07240_amd import workloads as W
from gpu_helpers import say, torch_cuda

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [300, 256, 40])
def test_answers(tokens):
    torch_cuda()
    from paper_2310_07240_amd import serving
    w = W.small(name="answers", n_ctx=2, n_layers=3, n_tokens=tokens, n_channels=256, chunk_len=128)
    r = serving.answer(w, kv_heads=4, q_heads=8, requests=5, drafts=3, steps=6, vocab=500)
    say(r)
    assert r["contexts"] == 6 and r["requests"] == 30 and r["tokens"] == tokens
    assert r["missing"] == 0 and 0 < r["accepted"] < 3
    # a code is off by at most half a step, 1 / 254 of its page's largest value (see test_serving_path)
    assert r["rel_error_8bit"] < 0.05 and r["rel_error_after"] < 0.05
    p = r["pages"]
    # only the contexts are left, whole and in front; while the requests ran, they shared them
    assert p["after"] == p["contexts"] == 6 * -(-tokens // 64)
    assert p["contexts"] < p["used"] <= p["contexts"] + 30 * 2
    assert tokens < 64 or p["used"] < p["unshared"]
    assert set(r["ms"]) == {"fork", "step", "verify", "release", "compact"}


def test_command(capsys, monkeypatch):
    torch_cuda()
    from paper_2310_07240_amd import serving
    w = W.small(name="answers", n_layers=2, n_tokens=100, n_channels=256, chunk_len=64)
    monkeypatch.setitem(W.WORKLOADS, "answers", w)
    assert serving.main(["--workload", "answers", "--heads", "4", "--q-heads", "4", "--requests", "3",
                         "--drafts", "1", "--steps", "2", "--vocab", "90"]) == 0
    r = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert r["requests"] == 6 and r["missing"] == 0
