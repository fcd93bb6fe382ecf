"""The conversation of examples/chat.py, short: what the cache holds, the bf16 path beside it, and the replayed steps."""
import importlib.util
import os

import pytest
import torch

from gpu_util import ensure_built

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("images", [False, True])
def test_a_short_conversation(images):
    ensure_built()
    spec = importlib.util.spec_from_file_location("chat", os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "chat.py"))
    chat = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(chat)
    lines = []
    turns, tokens, reply = 2, 200, 7
    a = chat.run(turns, tokens, reply, images, 3, lines.append)
    assert len(lines) == turns and a[0]["same"]
    # both paths round the turned values, the weights and the output to bf16 or more (2^-9 / sqrt 3 = 1.1e-3 of each): 5e-3 between them
    assert a[0]["off"] < 5e-3
    for t, r in enumerate(a):
        assert 0.2 < r["kept"] < 0.9 and torch.isfinite(r["out"].float()).all()
        assert len(r["replies"]) == reply and all(torch.isfinite(x.float()).all() for x in r["replies"])
        # sinks and replies are kept, and no more than everything
        assert all((t + 1) * (4 + reply) <= n <= (t + 1) * (tokens + reply) for n in r["rows"])
    b = chat.run(turns, tokens, reply, images, 3, lines.append)      # the same bits again
    for x, y in zip(a, b):
        assert torch.equal(x["out"], y["out"]) and all(torch.equal(p, q) for p, q in zip(x["replies"], y["replies"])) and x["rows"] == y["rows"]
