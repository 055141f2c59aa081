"""What the operators' entry points refuse of arrays that are in device memory, over a stand-in for the HIP runtime (tests/host_ops.cpp; no GPU needed)."""
import ctypes as C
import os
import random
import subprocess

import pytest

import paper_2412_11810_amd as snn
from paper_2412_11810_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2412_11810_amd", "csrc")


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    path = str(tmp_path_factory.mktemp("host_ops") / "host_ops.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-w", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I", CSRC, "-I", "/opt/rocm/include",
                    os.path.join(ROOT, "tests", "host_ops.cpp"), "-o", path], check=True)
    L = C.CDLL(path)
    ops.declare(L)
    return L


class Memory:
    """Addresses of arrays, 2^20 bytes apart (nothing is read there)."""

    def __init__(self, names):
        self.at = {name: (1 << 32) + (i << 20) for i, name in enumerate(names)}

    def __call__(self, **other):
        at = {**self.at, **{k: v if v is None or isinstance(v, int) else self.at[v] for k, v in other.items()}}
        return [at[name] for name in self.at]


def outcome(lib, call, *args):
    before = lib.launches()
    status = getattr(lib, call)(C.byref(ops.snn_launch(0, None, None, 0)), *args)
    assert status == snn.SNN_OK or lib.launches() == before
    return "" if status == snn.SNN_OK else (status, lib.snn_launch_error().decode())


def accepted(lib, call, *args, launches=1):
    before = lib.launches()
    assert outcome(lib, call, *args) == "" and lib.launches() == before + launches


def refused(lib, a, b, call, *args):
    status, text = outcome(lib, call, *args)
    assert status == snn.SNN_E_INVAL and f"{a} and {b} share elements" in text, text


FORWARD = Memory(["q", "k", "v", "g", "beta", "s0", "o", "s_last", "kept"])
BACKWARD = Memory(["q", "k", "v", "g", "beta", "kept", "do", "ds_last", "dq", "dk", "dv", "dg", "dbeta", "ds0"])
LENGTHS = 1 << 31


def delta(**k):
    return C.byref(ops.snn_delta(**{**dict(T=20, batch=2, heads=4, key_heads=2, dk=8, dv=4, dtype=0, scale=1.0, lengths=LENGTHS), **k}))


def test_results_of_the_delta_rule_share_nothing_with_other_arrays(lib):
    accepted(lib, "snn_delta_forward", delta(), *FORWARD())
    accepted(lib, "snn_delta_backward", delta(), *BACKWARD())
    for call, of, may in (("snn_delta_forward", FORWARD, {("o", "v"), ("s_last", "s0")}),
                          ("snn_delta_backward", BACKWARD, {("dq", "q"), ("dk", "k"), ("dv", "v"), ("dg", "g"), ("dbeta", "beta"), ("ds0", "ds_last")})):
        names = list(of.at)
        results = names[names.index("o" if call == "snn_delta_forward" else "dq"):]
        for i, a in enumerate(results):
            for b in names:
                if a == b:
                    continue
                if (a, b) in may:
                    accepted(lib, call, delta(), *of(**{a: b}))
                    at = of.at[b] + 4  # (but not a part of it)
                    refused(lib, a, b, call, delta(), *of(**{a: at}))
                else:
                    first, second = (a, b) if b not in results or results.index(b) > i else (b, a)
                    refused(lib, first, second, call, delta(), *of(**{a: b}))
            refused(lib, a, "lengths", call, delta(), *of(**{a: LENGTHS}))
    # their ends: q has 40 rows of 16 elements of 4 bytes, kept one of 2 * 4 * 8 * 4
    accepted(lib, "snn_delta_backward", delta(), *BACKWARD(dk=BACKWARD.at["q"] + 40 * 64))
    refused(lib, "dk", "q", "snn_delta_backward", delta(), *BACKWARD(dk=BACKWARD.at["q"] + 40 * 64 - 4))
    accepted(lib, "snn_delta_forward", delta(), *FORWARD(s0=FORWARD.at["kept"] + 1024))
    refused(lib, "kept", "s0", "snn_delta_forward", delta(), *FORWARD(s0=FORWARD.at["kept"] + 1020))
    refused(lib, "kept", "s0", "snn_delta_forward", delta(T=257), *FORWARD(s0=FORWARD.at["kept"] + 1024))
    # what is not there shares nothing
    accepted(lib, "snn_delta_forward", delta(T=0), *FORWARD(o="q", kept="s0"))
    accepted(lib, "snn_delta_backward", delta(), *BACKWARD(ds_last=None, ds0=None))


def test_parts_of_a_projection_are_apart(lib):
    # [T][batch][q 16, k 16, v 16, o 16] and their gradients; inputs and results in the rows of one array
    ld, base = 100, FORWARD.at["q"]
    p = dict(ld_q=ld, ld_k=ld, ld_v=ld, ld_o=ld, ld_dq=ld, ld_dk=ld, ld_dv=ld)
    accepted(lib, "snn_delta_forward", delta(**p), *FORWARD(q=base, k=base + 64, v=base + 128, o=base + 192))
    accepted(lib, "snn_delta_forward", delta(**p), *FORWARD(q=base, k=base + 64, v=base + 128, o=base + 128))
    accepted(lib, "snn_delta_forward", delta(**p), *FORWARD(q=base, k=base + 64, v=base + 128, o=base - 64))  # (the end of the row before)
    refused(lib, "o", "q", "snn_delta_forward", delta(**p), *FORWARD(q=base, k=base + 64, v=base + 128, o=base - 60))
    refused(lib, "o", "v", "snn_delta_forward", delta(**p), *FORWARD(q=base, k=base + 64, v=base + 128, o=base + 188))
    refused(lib, "o", "v", "snn_delta_forward", delta(**{**p, "ld_o": 2 * ld}), *FORWARD(q=base, k=base + 64, v=base + 128, o=base + 128))
    refused(lib, "o", "q", "snn_delta_forward", delta(**p), *FORWARD(q=base, k=base + 64, v=base + 128, o=base + 400))
    accepted(lib, "snn_delta_backward", delta(**p), *BACKWARD(do=base + 192, q=base, k=base + 64, v=base + 128, dq=base, dk=base + 64, dv=base + 128))
    refused(lib, "dv", "do", "snn_delta_backward", delta(**p), *BACKWARD(do=base + 192, q=base, k=base + 64, v=base + 128, dv=base + 192))


def test_a_step_by_itself_may_be_of_any_size(lib):
    # 2^26 bytes of v and o: chunks of 64 such steps would have places beyond 32 bits, a step forward has none
    for large in (dict(batch=1 << 18, dv=16), dict(ld_v=1 << 24), dict(ld_q=1 << 24), dict(ld_k=1 << 40)):
        def far(names):
            of = Memory(names)
            of.at = {name: i << 56 for i, name in enumerate(names, 1)}
            return of()
        accepted(lib, "snn_delta_forward", delta(T=1, **large), *far(FORWARD.at))
        for T, call, names in ((2, "snn_delta_forward", FORWARD.at), (0, "snn_delta_forward", FORWARD.at), (1, "snn_delta_backward", BACKWARD.at)):
            assert "2^25 bytes" in outcome(lib, call, delta(T=T, **large), *far(names))[1]
    assert "row to row" in outcome(lib, "snn_delta_forward", delta(T=1, ld_v=(1 << 40) + 1), *FORWARD())[1]
    assert "2^28" in outcome(lib, "snn_delta_forward", delta(T=1, batch=1 << 18, dv=257), *FORWARD())[1]


def test_results_of_the_norm_share_nothing_with_other_arrays(lib):
    p = dict(rows=10, n=40, dtype=0, eps=1e-6)
    norm = lambda **k: C.byref(ops.snn_norm(**{**p, **k}))  # noqa: E731
    forward, packed = Memory(["x", "residual", "w", "total", "y"]), Memory(["x", "residual", "w", "total", "the codes", "the exponents"])
    backward = Memory(["total", "w", "dy", "dtotal", "dx", "dw"])
    for call, of, results, may in (("snn_norm_forward", forward, ("total", "y"), {"total": ("x", "residual"), "y": ("x", "residual")}),
                                   ("snn_norm_forward_packed", packed, ("total", "the codes", "the exponents"), {"total": ("x", "residual")}),
                                   ("snn_norm_backward", backward, ("dx", "dw"), {"dx": ("total", "dy", "dtotal")})):
        accepted(lib, call, norm(), *of())
        for i, a in enumerate(results):
            for b in of.at:
                if a == b:
                    continue
                if b in may.get(a, ()):
                    accepted(lib, call, norm(), *of(**{a: b}))
                    refused(lib, a, b, call, norm(), *of(**{a: of.at[b] + 160}))  # (row on row only)
                else:
                    first, second = (a, b) if b not in results or results.index(b) > i else (b, a)
                    refused(lib, first, second, call, norm(), *of(**{a: b}))
    accepted(lib, "snn_norm_forward", norm(), *forward(total="x", y="residual"))
    accepted(lib, "snn_norm_forward", norm(), *forward(residual="x", total="x"))  # x + x
    refused(lib, "total", "y", "snn_norm_forward", norm(), *forward(total="x", y="x"))
    # the halves of wider rows, and rows that are not as far apart
    x = forward.at["x"]
    accepted(lib, "snn_norm_forward", norm(ld_x=80, ld_y=80), *forward(y=x + 160))
    refused(lib, "y", "x", "snn_norm_forward", norm(ld_x=80, ld_y=80), *forward(y=x + 156))
    refused(lib, "total", "x", "snn_norm_forward", norm(ld_x=40, ld_total=80), *forward(total=x))
    accepted(lib, "snn_norm_forward", norm(rows=1, ld_x=40, ld_total=80), *forward(total=x))
    accepted(lib, "snn_norm_forward", norm(rows=0), *forward(total="w"), launches=0)
    refused(lib, "dw", "w", "snn_norm_backward", norm(rows=0), *backward(dw="w"))


def test_what_a_step_of_adamw_writes_shares_nothing_with_other_arrays(lib):
    at = {name: (1 << 32) + (i << 20) for i, name in enumerate(("p", "g", "m", "v", "m_exps", "v_exps", "copy"))}
    step, scale = 1 << 30, (1 << 30) + 4

    def call(**k):
        how = ops.snn_adamw(1e-3, 0.9, 0.99, 1e-8, 0.1, 0, k.pop("step", step), k.pop("scale", scale))
        return "snn_adamw_step", C.byref(how), C.byref(ops.snn_adamw_tensor(**{**at, **dict(n=100), **k})), 1

    accepted(lib, *call())
    for a in at:
        for b in at:
            if a != b:
                assert "share" in outcome(lib, *call(**{a: at[b]}))[1], (a, b)
    size = dict(p=400, m=100, v=100, m_exps=4, v_exps=4, copy=200)
    for b, n in size.items():
        for one, what in (("step", "two of the arrays"), ("scale", "scale shares")):
            assert what in outcome(lib, *call(**{one: at[b] + (n - 1) // 4 * 4}))[1], (one, b)
            accepted(lib, *call(**{one: at[b] + (n + 3) // 4 * 4}))
    assert "scale shares" in outcome(lib, *call(scale=step))[1]
    accepted(lib, *call(scale=at["g"]))  # (which is only read)


def test_arrays_of_rows_share_memory_where_their_rows_do(tmp_path):
    source, exe = tmp_path / "share.cpp", str(tmp_path / "share")
    source.write_text("""#include "snn_share.h"
#include <stdio.h>
int main() {
  long long a, b, n[6];
  while (scanf("%lld %lld %lld %lld %lld %lld %lld %lld", &a, &n[0], &n[1], &n[2], &b, &n[3], &n[4], &n[5]) == 8)
    printf("%d", share(Rows{(void *)a, n[0], n[1], n[2]}, Rows{(void *)b, n[3], n[4], n[5]}));
}""")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC, str(source), "-o", exe], check=True)
    rng, cases = random.Random(1), []
    for _ in range(20000):
        x = []
        for _ in range(2):
            size = rng.randint(1, 9)
            x.append([100 + rng.randint(0, 60), rng.randint(0, 9), size, size + rng.randint(0, 3) * rng.randint(0, 6)])
        if rng.random() < 0.3:
            x[1][3] = max(x[1][2], x[0][3])
        cases.append(x)
    cover = lambda at, rows, size, step: {at + i * step + j for i in range(rows) for j in range(size)}  # noqa: E731
    want = [bool(cover(*a) & cover(*b)) for a, b in cases]
    # as large as arguments may be
    top = 1 << 42
    cases += [[[1 << 20, 1 << 40, 4, top], [1 << 20, 1 << 40, 4, top]], [[1 << 20, 1 << 40, 4, top], [(1 << 20) + 4, 1 << 40, 4, top]],
              [[1 << 20, 1 << 40, 4, top], [(1 << 20) + 4 * top, 1, 1, 1]], [[0, 5, 5, 5], [1, 5, 5, 5]]]
    want += [True, False, True, False]
    got = subprocess.run([exe], input="\n".join(" ".join(map(str, a + b)) for a, b in cases), capture_output=True, text=True, check=True).stdout
    assert [c == "1" for c in got] == want and 3000 < sum(want) < len(want) - 3000
