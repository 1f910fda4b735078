"""The host side of the experts' product on several devices, against a stand-in for the HIP runtime (CPU only): a kernel
is launched with more LDS than it may have by default only on devices where it was allowed to."""
import os
import subprocess

import pytest

from paper_2605_10670_amd import binding, build

ROOT = build.ROOT
F32, BF16, FP8 = binding.F32, binding.BF16, binding.FP8_E4M3
ALL_TYPES = [(x, y, gate) for x in (F32, BF16, FP8) for y, gate in ((F32, 0), (BF16, 0), (F32, 1), (BF16, 1), (FP8, 1))]

pytestmark = pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="needs hipcc")


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    at = tmp_path_factory.mktemp("product")
    objs = []
    for src in (os.path.join(build.HERE, "csrc", "product.hip"), os.path.join(ROOT, "tests", "product_host.cpp")):
        objs.append(str(at / (os.path.basename(src) + ".o")))
        subprocess.run([build.HIPCC, "--offload-arch=gfx950", "--cuda-host-only", "-O1", "-std=c++17", "-w", "-I", os.path.join(ROOT, "include"),
                        "-I", os.path.join(build.HERE, "csrc"), "-x", "hip", "-c", src, "-o", objs[-1]], check=True)
    # (the kernels' code, which is not there, is the one symbol left)
    subprocess.run(["g++", "-no-pie", *objs, "-Wl,--unresolved-symbols=ignore-all", "-o", str(at / "host")], check=True)

    def run(*lines):
        r = subprocess.run([str(at / "host")], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=60)
        assert r.returncode == 0, r.stderr
        return [tuple(line.split()) for line in r.stdout.splitlines()]
    return run


def large(events):
    """(device, kernel, LDS bytes) of the launches that need a kernel's own limit."""
    return [(e[1], e[2], int(e[5])) for e in events if e[0] == "launch" and int(e[5]) > 65536]


def results(events):
    return [int(e[1]) for e in events if e[0] in ("create", "run", "destroy")]


@pytest.mark.parametrize("x,y,gate", ALL_TYPES)
def test_every_device_is_asked(host, x, y, gate):
    lines = []
    for device in (0, 3):
        lines += [f"device {device}", f"create p{device} 1 1024 1024 {x} {y} {gate} 20000"]
    for device in (3, 0):
        lines.append(f"device {device}")
        lines += [f"run p{device} {rows} 0" for rows in (200, 8192, 20000)]
    events = host(*lines)
    assert results(events) == [binding.OK] * 8
    allowed = {}
    for e in events:
        if e[0] == "attribute":
            allowed[e[1], e[2]] = int(e[3])
        for device, kernel, lds in large([e]):
            assert allowed.get((device, kernel), 65536) >= lds, f"device {device}: {kernel} may not have {lds} bytes"
    assert {d for d, _, _ in large(events)} == {"0", "3"}


def test_a_failure_is_not_kept(host):
    """A device that refuses once: the handle is not made, the next one is, and works."""
    events = host("fail 1", f"create p 1 1024 1024 {BF16} {BF16} 0 4096", f"create q 1 1024 1024 {BF16} {BF16} 0 4096", "run q 4096 0")
    assert results(events) == [binding.ERR_HIP, binding.OK, binding.OK]
    assert large(events)


@pytest.mark.parametrize("x,y,gate", ALL_TYPES)
def test_a_workspace_for_codes_only(host, x, y, gate):
    """What the kernel of few rows hands from one workgroup to another are the values behind codes."""
    events = host("device 2", f"create p 1 1024 1024 {x} {y} {gate} 16", "run p 16 0", "destroy p")
    assert results(events) == [binding.OK] * 3
    kinds = [e[0] for e in events]
    assert kinds.count("malloc") == kinds.count("free") == (1 if y == FP8 else 0)
    assert all(e[1] == "2" for e in events if e[0] in ("malloc", "free"))
