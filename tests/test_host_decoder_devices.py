"""The device that is current when decoder.py's calls reach the library: the tensors', whichever the caller's is (no GPU: the calls are compiled around stand-ins, and run in a process of their own)."""
import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

BODY = """
import ctypes, importlib.util, sys
sys.path.insert(0, {root!r})
import torch
import paper_2007_12216_amd as rn
def load(name):
    spec = importlib.util.spec_from_file_location(name, {path!r})
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module
stand_in, call = load("decoder_devices"), load("_decoder")
cache = rn.Cache4Desc(1 << 20, 1 << 20, 1 << 20, 1 << 20, 10, 16, 2, 128)
rope = rn.RopeDesc(q_heads=4, kv_heads=2, head_dim=128, rotary=128, max_position=100, eps=1e-6)
attention = rn.AttentionDesc(q_heads=4, scale=0.1)
address = ctypes.addressof
def calls(d):
    make = lambda *a: stand_in.make(d, *a)
    i = lambda n: make("int", n)
    k = make("byte", 10, 2, 16, 64)
    return dict(tables=lambda: call.tables(i(3), i(3), i(9), make("int", 3, 8), i(4), i(3), make("long", 5), i(5), i(1), 16),
                rope=lambda: call.rope(address(rope), make("float", 100, 128), None, None, make("bf16", 5, 768), i(5)),
                append=lambda: call.append(address(rope), make("float", 100, 128), None, None, make("bf16", 5, 1024), i(5), make("long", 5), address(cache), *CACHE(k)),
                read=lambda: call.read(address(cache), make("long", 5), 0, *CACHE(k)),
                attend=lambda: call.attend(address(cache), address(attention), make("bf16", 5, 4, 128), make("int", 3, 7), i(3), i(4), 0, 0, None, None, [], *CACHE(k)),
                linear=lambda: call.linear(make("byte", 64, 384), make("float", 1, 3), 300, make("bf16", 5, 300), None, None, []))
"""


def module(folder):
    from paper_2007_12216_amd.build import CSRC, extension_command
    path = os.path.join(folder, "decoder_devices.so")
    cmd = [os.path.join(ROOT, "tests", "host", "decoder_devices.cpp") if a.endswith("decoder_binding.cpp") else a for a in extension_command(path) if not a.startswith("-l:")]
    done = subprocess.run([*cmd[:1], "-I" + CSRC, *cmd[1:], "-L" + os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "lib"), "-lamdhip64"], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert done.returncode == 0, done.stdout[-3000:]
    return path


@pytest.fixture(scope="module")
def child(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    path = module(str(tmp_path_factory.mktemp("devices")))

    def run(body, cache="()"):
        done = subprocess.run([sys.executable, "-c", BODY.format(root=ROOT, path=path).replace("CACHE(k)", cache) + body], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
        assert done.returncode == 0, done.stdout[-3000:]
    return run


def test_calls_are_made_on_their_tensors_device(child):
    child("""
for d in (0, 1, 5):
    for name, f in calls(d).items():
        f()
        assert stand_in.launches() == [f"{name} on {d}, stream of {d}"], (name, d)
        assert stand_in.current() == 0
""")


def test_a_cache_on_another_device_is_refused(child):
    child("""
f = calls(1)
for name in ("append", "read", "attend"):
    try:
        f[name]()
        raise SystemExit(f"{name}: not refused")
    except ValueError as e:
        assert "cache must be on" in str(e), (name, e)
assert stand_in.launches() == [] and stand_in.current() == 0
""", cache="(stand_in.make(0, 'byte', 10, 2, 16, 64),)")
    child("""
for name in ("append", "read", "attend"):
    calls(3)[name]()
assert [s.split(",")[0] for s in stand_in.launches()] == ["append on 3", "read on 3", "attend on 3"]
""", cache="(k,)")


def test_objects_over_several_devices_are_refused(child):
    child("""
torch.cuda.is_available = lambda: True
from paper_2007_12216_amd import decoder
def refused(f, name):
    try:
        f()
    except ValueError as e:
        assert f"{name} must be" in str(e) and "cuda:1" in str(e), e
        return
    raise SystemExit(f"{name}: not refused")
shapes = [(10, 2, 16, 64), (10, 2, 16, 4)] * 2
for other in (None, 1, 2, 3):
    tensors = [stand_in.make(0 if i == other else 1, "byte", *s) for i, s in enumerate(shapes)]
    make = lambda: decoder.Cache4(10, 16, 2, 128, tensors=tensors)
    if other is None:
        assert str(make().device) == "cuda:1"
    else:
        refused(make, ("k", "k_scale", "v", "v_scale")[other])
decoder.Fp8Linear(stand_in.make(1, "byte", 64, 384), stand_in.make(1, "float", 1, 3), 300)
refused(lambda: decoder.Fp8Linear(stand_in.make(1, "byte", 64, 384), stand_in.make(0, "float", 1, 3), 300), "scales")
""")
