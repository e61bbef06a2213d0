"""Host side of the operators by which compressed models are judged and tuned under AddressSanitizer and
UndefinedBehaviorSanitizer: no device code is built, nothing runs on a GPU."""
import os
import shutil
import subprocess

import pytest

from .test_sanitizers import ENV, ROOT, SAN, _run


def test_operators_host_side_under_sanitizers(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("no hipcc")
    csrc = os.path.join(ROOT, "paper_2208_11580_amd", "csrc")
    objs, procs = [], []
    for name in ("ctx", "global_select", "score", "layernorm", "embed", "adamw"):
        obj = str(tmp_path / (name + ".o"))
        objs.append(obj)
        procs.append((name, subprocess.Popen([hipcc, "--offload-host-only", "-std=c++17", "-fPIC"] + SAN +
                                             ["-c", os.path.join(csrc, name + ".hip"), "-o", obj],
                                             stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    for name, p in procs:
        out, _ = p.communicate()
        assert p.returncode == 0, "%s\n%s" % (name, out[-3000:])
    # stand-ins for the device images that the full build embeds
    undef = set()
    for obj in objs:
        undef |= {ln for ln in _run(["nm", "-u", obj]).stdout.split() if ln.startswith("__hip_fatbin_")}
    stub = str(tmp_path / "stubs.c")
    with open(stub, "w") as f:
        for name in sorted(undef):
            f.write("const unsigned char %s[64] __attribute__((aligned(4096))) = {0};\n" % name)
    lib = str(tmp_path / "libobc_tuning_host.so")
    _run([hipcc, "--offload-host-only", "-shared", "-fPIC"] + SAN + ["-o", lib] + objs + ["-x", "c", stub])
    exe = str(tmp_path / "tuning_host_san")
    clangxx = os.path.join(os.path.dirname(os.path.realpath(hipcc)), "..", "lib", "llvm", "bin", "clang++")
    if not os.path.exists(clangxx):
        clangxx = shutil.which("clang++") or "/opt/rocm/lib/llvm/bin/clang++"
    _run([clangxx, "-std=c++17"] + SAN + ["-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "sanitize", "tuning_host_main.cpp"),
                                          "-o", exe, "-L", str(tmp_path), "-lobc_tuning_host", "-Wl,-rpath," + str(tmp_path)])
    r = _run([exe], env=ENV)
    assert "operators' host sanitizer run clean" in r.stdout
