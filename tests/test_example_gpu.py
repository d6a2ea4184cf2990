"""The example that takes image tokens to generated tokens runs and checks itself."""
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_kept_tokens_prefill():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA GPU")
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "kept_tokens_prefill.py"), "--images", "2",
                        "--tokens", "3"], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert "match" in r.stdout
