"""Host-side sanitizer pass (no GPU) over the mixture-of-experts and AdamW entry points: argument validation, workspace planning and
the AdamW table under AddressSanitizer + UndefinedBehaviorSanitizer, with kernel launchers that check the places they are given."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_host_layer_under_sanitizers_with_stubbed_launchers(tmp_path):
    csrc, exe = os.path.join(ROOT, "paper_2507_16099_amd", "csrc"), str(tmp_path / "moe_sanitize_check")
    r = subprocess.run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++20",
                        "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all",
                        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument", "-o", exe,
                        os.path.join(ROOT, "tests", "moe_sanitize_check.hip"), os.path.join(csrc, "moe_api.hip"), os.path.join(csrc, "adamw.hip"),
                        os.path.join(csrc, "tuning.hip")],
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    # the HIP runtime keeps process-lifetime allocations: leak checking off, everything else on
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600, env={**os.environ, "ASAN_OPTIONS": "detect_leaks=0"})
    assert r.returncode == 0 and "moe_sanitize_check ok" in r.stdout, f"{r.stdout[-3000:]}\n{r.stderr[-3000:]}"
