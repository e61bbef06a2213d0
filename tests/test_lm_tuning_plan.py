"""AdamW's plan refuses arrays that a step must not share: the host side under AddressSanitizer and UndefinedBehaviorSanitizer, no
device code, nothing on a GPU."""
import os

import pytest

from .test_sanitizers import ENV, ROOT, SAN, _run


def test_plans_refuse_arrays_that_overlap(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    csrc = os.path.join(ROOT, "paper_2208_11580_amd", "csrc")
    objs = []
    for name, src in (("adamw", os.path.join(csrc, "adamw.hip")), ("main", os.path.join(ROOT, "tests", "sanitize", "plan_host_main.cpp"))):
        objs.append(str(tmp_path / (name + ".o")))
        _run([hipcc, "--offload-host-only", "-x", "hip", "-std=c++17", "-fPIC"] + SAN + ["-c", src, "-o", objs[-1]])
    # stand-ins for the device images that the full build embeds
    undef = {ln for obj in objs for ln in _run(["nm", "-u", obj]).stdout.split() if ln.startswith("__hip_fatbin_")}
    stub = str(tmp_path / "stubs.c")
    with open(stub, "w") as f:
        for name in sorted(undef):
            f.write("const unsigned char %s[64] __attribute__((aligned(4096))) = {0};\n" % name)
    exe = str(tmp_path / "plan_host_san")
    _run([hipcc, "--offload-host-only"] + SAN + ["-o", exe] + objs + ["-x", "c", stub])
    r = _run([exe], env=ENV)
    assert "plan's host sanitizer run clean" in r.stdout
