"""GPU: the serving example's prompts in pieces and replayed decode steps, against FP32 attention over the cache read
back (bfloat16 outputs: a relative error of 2^-9 in the mean square, 2^-8 at most)."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "kv4_serving.py")


@pytest.mark.parametrize("model,seqs,prompt,steps", [("1.5b", 3, 300, 9), ("7b", 2, 64, 70)])
def test_serving_example(model, seqs, prompt, steps):
    spec = importlib.util.spec_from_file_location("kv4_serving", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    print("example", model, seqs, prompt, steps, flush=True)
    assert mod.main(["--model", model, "--seqs", str(seqs), "--prompt", str(prompt), "--steps", str(steps)]) < 2.0 ** -8
