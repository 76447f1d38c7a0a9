"""The entry points of the layer, the loss and the AdamW step under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only):
tests/sanitize/train_driver.cpp walks random arguments through all of them, built without kernels, and compares every status with the documented rules."""
import os
import subprocess


def test_training_entry_points_are_clean_under_address_and_ub_sanitizers():
    from paper_2011_06295_amd import build as libbuild
    exe = libbuild.build_sanitize_train()
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    res = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=600)
    assert res.returncode == 0, res.stdout[-4000:]
    assert "train driver: ok" in res.stdout and "runtime error" not in res.stdout
