"""As test_host_share_sanitizers.py, with every piece of the shared attention's workspace checked (tests/host_sanitize/share_sizes_driver.hip)."""
import os
import shutil
import subprocess

import pytest

from test_host_sanitizers import BUILD, COMMAND, ROOT

EXE = os.path.join(BUILD, "host_share_sizes_sanitized")


def test_every_piece_of_the_shared_workspace_lies_in_it():
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc not available")
    os.makedirs(BUILD, exist_ok=True)
    command = [x.replace("driver.hip", "share_sizes_driver.hip") for x in COMMAND[:-1]] + [EXE]
    for name in ("cache_api.hip", "share_api.hip"):
        command.insert(command.index("-o"), os.path.join(ROOT, "paper_2502_04077_amd", "csrc", name))
    res = subprocess.run(command, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([EXE], capture_output=True, text=True, env=env, timeout=300)
    assert run.returncode == 0, (run.stdout + run.stderr)[-3000:]
    assert "all checks passed" in run.stdout
    assert "AddressSanitizer" not in run.stderr and "runtime error" not in run.stderr
