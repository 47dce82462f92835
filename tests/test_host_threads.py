"""What the library remembers of a device between calls may be asked and set by any host thread: built with the compiler's
thread sanitizer, on the CPU."""
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
        # where the sanitizer is missing or does not run, the program still has to build
        subprocess.run([c for c in cmd if c != "-fsanitize=thread"], check=True)
    return str(exe)


def test_flags_of_devices_are_free_of_races(tmp_path):
    out = subprocess.run([build(tmp_path, PROGRAM, "flags")], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and out.stdout == "done\n", out.stdout + out.stderr


def test_the_sanitizer_sees_a_plain_word(tmp_path):
    """The mistake planted: the same program on a class without atomics."""
    plain = PROGRAM.replace('#include "device_flags.h"', """namespace modse { struct DeviceFlags {
        unsigned long long bits = 0;
        bool has(int d) const { return d >= 0 && d < 64 && ((bits >> d) & 1); }
        void set(int d) { if (d >= 0 && d < 64) bits |= 1ull << d; } }; }""")
    out = subprocess.run([build(tmp_path, plain, "plain")], capture_output=True, text=True, timeout=120)
    if "ThreadSanitizer" not in out.stderr:
        pytest.skip("no thread sanitizer here")
    assert "data race" in out.stderr


def test_no_source_keeps_such_a_word_plain():
    """Plain statics that a call writes: none beside the debugging switches, which are set between calls."""
    import re
    for name in sorted(os.listdir(CSRC)):
        text = open(os.path.join(CSRC, name)).read()
        for line in re.findall(r"^ +static (?:unsigned|int|bool|long|size_t|[A-Z]\w*Fn)\b[^(\n]*[;{].*$", text, re.M):
            assert "constexpr" in line or "const " in line, (name, line)


@pytest.mark.gpu
def test_a_threads_first_call_of_each_operator():
    """A host thread has no current context until a call gives it one; any operator may be that call."""
    import threading
    torch = pytest.importorskip("torch")
    from paper_2409_12210_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(0)
    mk = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    ws = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")
    d, V, widths = 256, 3000, (128, 384)
    S = sum(widths)
    layer, w = B.ModseLayer(d, widths, 1), (mk(2, d), mk(S, d), mk(S, d), mk(d, S))
    calls = []
    for T in (4, 20, 300):
        x, lab, f = mk(T, d), torch.randint(0, V, (T,), generator=g, device="cuda"), lambda: torch.zeros(T, device="cuda")
        head, y, z, loss, lse, dx, dw = mk(V, d), mk(T, V), mk(T, V), f(), f(), mk(T, d), mk(V, d)
        a = ws(B.linear_workspace_bytes(torch.bfloat16, T, d, V)), ws(B.linear_backward_workspace_bytes(T, d, V))
        c = ws(B.cross_entropy_workspace_bytes(T, d, V)), ws(B.cross_entropy_backward_workspace_bytes(T, d, V))
        e, out, table = ws(B.embedding_backward_workspace_bytes(T, d, V)), mk(T, d), mk(V, d)
        calls += [(lambda x=x, head=head, y=y, a=a: B.linear(x, head, y, a[0]), [y]),
                  (lambda x=x, head=head, lab=lab, loss=loss, lse=lse, c=c: B.cross_entropy(x, head, lab, loss, lse, c[0]), [loss, lse]),
                  (lambda x=x, head=head, lab=lab, lse=lse, dx=dx, dw=dw, c=c: B.cross_entropy_backward(x, head, lab, lse, dx, dw, c[1]), [dx, dw]),
                  (lambda lab=lab, table=table, out=out: B.embedding(lab, table, out), [out]),
                  (lambda lab=lab, x=x, table=table, e=e: B.embedding_backward(lab, x, table, e), [table])]
        fw, yl = layer.alloc_workspace(torch.bfloat16, T, False), mk(T, d)
        calls.append((lambda x=x, yl=yl, fw=fw: layer.forward(*w, x, yl, fw, False), [yl]))
        if T <= 32:
            dws, yd = layer.alloc_decode_workspace(torch.bfloat16, T), mk(T, d)
            calls.append((lambda x=x, yd=yd, dws=dws: layer.decode(*w, x, yd, dws), [yd]))
    up, grad = torch.empty(256, 512, dtype=torch.bfloat16, device="cuda"), mk(256, 512)
    ows = ws(B.orthogonalize_workspace_bytes([(256, 512)]))
    calls.append((lambda: B.orthogonalize([grad], [up], ows), [up]))
    torch.cuda.synchronize()
    failed = []

    def work(call):
        try:
            call()
        except Exception as e:                       # shown by the assertion below
            failed.append((e, call))
    for call, outs in calls:
        call()
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        t = threading.Thread(target=work, args=(call,))
        t.start()
        t.join()
        torch.cuda.synchronize()
        assert not failed and all(torch.equal(a, b) for a, b in zip(want, outs)), failed
    layer.destroy()
