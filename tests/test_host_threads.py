"""What the library remembers of a device between calls may be asked and set by any host thread: built with the compiler's
thread checker, on the CPU."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2409_12210_b200", "csrc")
PROGRAM = r"""
#include "device_flags.h"
#include <cstdio>
#include <thread>
#include <vector>
static modse::DeviceFlags flags;
int main()
{
    std::vector<std::thread> all;
    for (int t = 0; t < 8; ++t)
        all.emplace_back([t] {
            for (int i = 0; i < 70; ++i) {
                const int device = (i + 9 * t) % 70 - 2;
                if (!flags.has(device)) flags.set(device);
                if (flags.has(device) != (device >= 0 && device < 64)) std::puts("lost");
            }
        });
    for (auto &t : all) t.join();
    for (int d = 0; d < 64; ++d)
        if (!flags.has(d)) std::puts("lost");
    std::puts("done");
}
"""


def build(tmp_path, source, name):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    src, exe = tmp_path / (name + ".cc"), tmp_path / name
    src.write_text(source)
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-pthread", "-fsanitize=thread", "-I", CSRC, str(src), "-o", str(exe)]
    made = subprocess.run(cmd, capture_output=True).returncode == 0
    if not made or "FATAL: ThreadSanitizer" in subprocess.run([str(exe)], capture_output=True, text=True, timeout=120).stderr:
        # where the checker is missing or does not run, the program still has to build
        subprocess.run([c for c in cmd if c != "-fsanitize=thread"], check=True)
    return str(exe)


def test_flags_of_devices_are_free_of_races(tmp_path):
    out = subprocess.run([build(tmp_path, PROGRAM, "flags")], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and out.stdout == "done\n", out.stdout + out.stderr


def test_the_checker_sees_a_plain_word(tmp_path):
    """The mistake planted: the same program on a class without atomics."""
    plain = PROGRAM.replace('#include "device_flags.h"', """namespace modse { struct DeviceFlags {
        unsigned long long bits = 0;
        bool has(int d) const { return d >= 0 && d < 64 && ((bits >> d) & 1); }
        void set(int d) { if (d >= 0 && d < 64) bits |= 1ull << d; } }; }""")
    out = subprocess.run([build(tmp_path, plain, "plain")], capture_output=True, text=True, timeout=120)
    if "ThreadSanitizer" not in out.stderr:
        pytest.skip("no thread checker here")
    assert "data race" in out.stderr


def test_no_source_keeps_such_a_word_plain():
    """Plain statics that a call writes: none beside the debugging switches, which are set between calls."""
    import re
    for name in sorted(os.listdir(CSRC)):
        text = open(os.path.join(CSRC, name)).read()
        for line in re.findall(r"^ +static (?:unsigned|int|bool|long|size_t|[A-Z]\w*Fn)\b[^(\n]*[;{].*$", text, re.M):
            assert "constexpr" in line or "const " in line, (name, line)
