"""Which workgroup of an attention call has which task (csrc/decode.hpp), with the host compiler."""
import os

from test_sanitize_host import CSRC, ROOT, build_and_run


def test_every_task_once(tmp_path):
    t = os.path.join(ROOT, "tests")
    build_and_run(tmp_path, "g++", ["-std=c++17", "-Wall", "-I", os.path.join(t, "stub_wavefronts"), "-I", os.path.join(ROOT, "include"), "-I", CSRC],
                  [os.path.join(t, "host_dealt_out.cpp")], "dealt_out")
