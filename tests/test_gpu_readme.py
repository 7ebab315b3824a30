"""The README's Python example runs as it stands."""
import pathlib
import re

import pytest
import torch

from _gpu import say

pytestmark = pytest.mark.gpu


def test_the_example_of_sampled_generation():
    text = (pathlib.Path(__file__).resolve().parents[1] / "README.md").read_text()
    code, = re.findall(r"```python\n(.*?)```", text, flags=re.S)
    say("[readme] example")
    names = {}
    exec(code, names)
    torch.cuda.synchronize()
    assert (names["token"] >= 0).all() and (names["token"] < names["V"]).all()
    assert (names["logprob"] <= 0).all() and torch.isfinite(names["out"]).all()
    assert names["kv_len"].tolist() == [101] * names["R"]
