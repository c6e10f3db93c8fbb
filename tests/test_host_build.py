"""What the builds run, and that every library they make has all entry points."""
import os
import subprocess
import sys

import paper_2006_10901_amd as spdl
from paper_2006_10901_amd import build


def test_every_compile_and_link_command_is_hipcc(monkeypatch):
    """The C library alone: one compile per source, however it is started, and the link.  Nothing is compiled here."""
    ran = []

    class Started:
        returncode = 0

        def __init__(self, cmd, **kw):
            ran.append(cmd)

        def communicate(self):
            return "", None

    monkeypatch.setattr(subprocess, "Popen", Started)
    monkeypatch.setattr(subprocess, "run", lambda cmd, **kw: ran.append(cmd) or subprocess.CompletedProcess(cmd, 0, ""))
    monkeypatch.setattr(build.loads_in_flight, "check", lambda *a: 8)
    assert build.build_library() == build.LIB_PATH
    assert len(ran) == len(build.sources()) + 1 and all(cmd[0] == build.HIPCC for cmd in ran)
    for cmd, source in zip(ran, build.sources()):
        assert source in cmd and "-c" in cmd and "--offload-arch=gfx950" in cmd and "-packed-fp32-ops" in cmd
        assert all(flag in cmd for flag in build.SOURCE_FLAGS.get(os.path.basename(source), []))
    assert "-shared" in ran[-1] and build.LIB_PATH in ran[-1]
    ran.clear()
    assert build.build_phase_clocks() == build.CLOCKS_LIB_PATH
    assert all(cmd[0] == build.HIPCC for cmd in ran)
    assert [s for cmd, s in zip(ran, build.sources()) if s in cmd and "-DSPDL_PHASE_CLOCKS" in cmd] == build.sources()


def test_the_copy_with_clocks_is_a_library_that_the_binding_takes():
    """microbench/phase_clocks.py puts it in the library's place before the first call."""
    if not os.path.exists(build.CLOCKS_LIB_PATH):
        build.build_phase_clocks()
    program = ("from paper_2006_10901_amd import binding, build\n"
               "binding.LIB_PATH = build.CLOCKS_LIB_PATH\n"
               "import paper_2006_10901_amd as spdl\n"
               "lib = binding.lib()\n"
               "assert lib.spdl_debug_phase_clocks\n"
               "print(spdl.spdl_version(), spdl.spdl_attention_mask_bytes(1, 1))\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", program], cwd=root, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert done.returncode == 0, done.stdout
    assert done.stdout.split()[-2:] == [str(spdl.spdl_version()), str(8 * (64 + 64 + 1 + 1))]
