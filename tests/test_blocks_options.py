"""Options of the learned-feature model that need no GPU."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("options", [dict(types=4), dict(dropout=0.1), dict(types=0, blocks=1), dict(blocks=-1), dict(blocks=1, dropout=1.5)])
def test_options_without_an_effect_are_refused(options):
    from paper_2506_20818_b200.learned_features import LearnedFeatures
    with pytest.raises(ValueError):
        LearnedFeatures(None, 100, **options)


@pytest.mark.parametrize("options", [["--types", "4"], ["--dropout", "0.1"], ["--types", "2", "--dropout", "0.1"]])
def test_the_command_refuses_them_too(options):
    done = subprocess.run([sys.executable, "-m", "paper_2506_20818_b200.learned_features", *options], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert done.returncode == 2 and "--blocks" in done.stderr
