"""What a launch raises once for a kernel (csrc/per_device.h) is raised on every device that the process uses, on the host: the file itself compiled by the host compiler, with
a runtime of two and more devices in place of the GPU's."""
import glob
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2302_00282_amd", "csrc")

PROGRAM = r"""
#include <set>
#include <stdio.h>
#include <utility>
typedef int hipError_t;
enum { hipSuccess = 0, hipErrorInvalidValue = 1, hipFuncAttributeMaxDynamicSharedMemorySize = 8 };
static int current = 0, calls = 0, refuse = 0, bytes_asked = 0;
static std::set<std::pair<int, const void*>> limits;
static hipError_t hipGetDevice(int* d) { *d = current; return current < 0 ? hipErrorInvalidValue : hipSuccess; }
static hipError_t hipFuncSetAttribute(const void* f, int, int bytes) {
  ++calls, bytes_asked = bytes;
  if (refuse) return hipErrorInvalidValue;
  limits.insert({current, f});
  return hipSuccess;
}
#include "per_device.h"
using namespace xenos;

static void kernel_a(int) {}
static void kernel_b(int) {}
static int bad = 0;
static void is(bool ok, const char* what) {
  if (!ok) ++bad, printf("wrong: %s\n", what);
}
// (a kernel's first launch, or a later one)
static hipError_t launch_a(int device) {
  static PerDevice raised;
  current = device;
  const hipError_t e = raise_lds_limit(kernel_a, raised);
  if (e == hipSuccess) is(limits.count({device, (const void*)kernel_a}), "a launch on a device whose limit is as it was");
  return e;
}
static hipError_t launch_b(int device) {
  static PerDevice raised;
  current = device;
  return raise_lds_limit(kernel_b, raised, 70000);
}

int main() {
  for (int turn = 0; turn < 3; ++turn)
    for (int device : {0, 1, 7, 63, 64, 100}) is(launch_a(device) == hipSuccess, "success");
  is(bytes_asked == 160 * 1024, "all of a unit's memory");
  is(calls == 4 + 3 * 2, "once a device, each time beyond the 64th");
  refuse = 1, calls = 0;
  is(launch_b(2) == hipErrorInvalidValue && launch_b(2) == hipErrorInvalidValue && calls == 2, "a refusal is handed on and not taken for done");
  refuse = 0;
  is(launch_b(2) == hipSuccess && launch_b(2) == hipSuccess && calls == 3 && bytes_asked == 70000, "then done");
  is(launch_a(-1) != hipSuccess, "no device");
  return bad != 0;
}
"""


def test_a_limit_is_raised_once_on_each_device(tmp_path):
    src, exe = tmp_path / "per_device.cpp", tmp_path / "per_device"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr


def test_every_launcher_raises_it_this_way():
    for path in glob.glob(os.path.join(CSRC, "*")):
        if path.endswith((".hip", ".cpp", ".h")):
            with open(path) as f:
                text = f.read()
            assert os.path.basename(path) == "per_device.h" or "hipFuncSetAttribute" not in text, path
            # each call next to a flag of its own
            assert len(re.findall(r"static PerDevice raised;\n(?:.*\n)?.* raise_lds_limit\(", text)) == len(re.findall(r" raise_lds_limit\((?!F\*)", text)), path
