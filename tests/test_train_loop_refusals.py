"""What the training loop refuses, before it touches a device."""
import pathlib
import subprocess
import sys

import pytest

from paper_1804_08066_b200 import train_loop


def test_norm_without_rows_to_normalise():
    with pytest.raises(ValueError, match="norm"):
        train_loop.run(iters=1, model="cnn", norm=True)


def test_norm_without_rows_to_normalise_on_the_command_line():
    root = pathlib.Path(__file__).resolve().parent.parent
    for model in ([], ["--model", "cnn"]):
        r = subprocess.run([sys.executable, "-m", "paper_1804_08066_b200.train_loop", "--iters", "1", "--norm", *model], cwd=root,
                           capture_output=True, text=True, timeout=300)
        assert r.returncode == 2 and "--norm needs --model tokens" in r.stderr
