"""The arguments of serving_step.py's measurements of the paged cache."""
import json
import sys

import pytest

import serving_step


@pytest.mark.parametrize("given, steps", [([], 64), (["--decode", "128"], 128), (["--decode", "1"], 1), (["--decode", "30"], 30)])
def test_steps_as_asked_for(monkeypatch, given, steps):
    seen = []
    monkeypatch.setattr(serving_step, "paged_attention", lambda *a: seen.append(a))
    monkeypatch.setattr(sys, "argv", ["serving_step.py", "--paged-attention", *given])
    serving_step.main()
    assert seen == [(16, 8, 8192, 32, 32, 128, 1, steps)]
    monkeypatch.setattr(serving_step, "hybrid", lambda *a: seen.append(a))
    monkeypatch.setattr(sys, "argv", ["serving_step.py", "--hybrid", *given])
    serving_step.main()
    assert seen[1][-1] == (int(given[1]) if given else 128)


@pytest.mark.gpu
@pytest.mark.parametrize("drafted", [1, 5])
def test_a_single_step(capsys, drafted):
    serving_step.paged_attention(1, 2, 100, 4, 2, 64, drafted, 1)
    line = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert line["status"] == 0 and line["eager_us"] > 0 and line["graph_us"] > 0
