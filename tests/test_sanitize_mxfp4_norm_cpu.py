"""CPU: the refusals of MXFP4 caches, of reading back and of the norms under AddressSanitizer and UndefinedBehaviorSanitizer."""
import subprocess
import sys

from tests.test_sanitize_cpu import ROOT, sanitized_env  # noqa: F401 (a fixture)


def test_refusals_under_asan_and_ubsan(sanitized_env):  # noqa: F811
    env, _ = sanitized_env
    cmd = [sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider", "-m", "not gpu", "tests/test_mxfp4_norm_abi_cpu.py"]
    p = subprocess.run(cmd, env=env, cwd=ROOT, capture_output=True, text=True, timeout=900)
    out = p.stdout + p.stderr
    assert p.returncode == 0, out[-4000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out and " passed" in out, out[-4000:]
