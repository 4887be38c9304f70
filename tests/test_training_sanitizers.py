"""Host code of the calls that train device levels by reward under AddressSanitizer and UndefinedBehaviorSanitizer:
checks of arguments, sizes of launches, and the lists of tensors that a launch takes as its argument."""

import os
import subprocess

from test_sanitizers import CSRC, ENV, HERE, _compile, _link, hipcc  # noqa: F401


def test_training_host_paths_under_sanitizers(hipcc, tmp_path):  # noqa: F811
    objs = [_compile(hipcc, src, str(tmp_path / f"u{i}.o")) for i, src in enumerate(
        (os.path.join(CSRC, "api.hip"), os.path.join(CSRC, "kernels.hip"),
         os.path.join(HERE, "native", "training_host_check.cpp")))]
    exe = tmp_path / "training_host_check"
    # (the pass kernels' units are not called and not linked)
    cmd = [*_link(hipcc, objs, exe), "-Wl,--unresolved-symbols=ignore-all"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=600, env=ENV)
    assert out.returncode == 0, (out.stdout + out.stderr)[-6000:]
    assert "ALL OK" in out.stdout
    assert "runtime error" not in out.stderr
