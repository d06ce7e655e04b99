"""Device functions of the attention's headers as host code, under the checks of undefined arithmetic
(no GPU): hipcc compiles them for both sides, and only the host's runs."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
SRC = r'''
#include <cstdio>
#include <hip/hip_runtime.h>
#pragma clang force_cuda_host_device begin
#include "%s"
#pragma clang force_cuda_host_device end
using namespace dro;
int main()
{
%s
}
'''


def run(tmp_path, header, body):
    """What a program prints whose main is `body`, with `header` included; an operation without a
    defined result ends it."""
    src, exe = tmp_path / "t.hip", tmp_path / "t"
    src.write_text(SRC % (header, body))
    subprocess.run([HIPCC, "-std=c++17", "-O1", "--cuda-host-only",
                    "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all",
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2607_16892_amd", "csrc"),
                    str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return r.stdout
