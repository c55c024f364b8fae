"""What the C entry points launch, without a GPU: the calls are made in a process of their own, in which the kernel launch only writes down its arguments."""
import json
import os
import re
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
P = 0x10000  # an address that is never dereferenced

CHILD = """
import ctypes, json, sys
log = ctypes.CDLL(sys.argv[1]).launch_log
log.restype = ctypes.c_char_p
import paper_2604_12798_amd as vfa
L = vfa.lib()
out = []
for name, args, head in json.load(sys.stdin):
    log(head)
    f = getattr(L, name)
    rc = f(*[ctypes.c_void_p(a) if t is ctypes.c_void_p else a for a, t in zip(args, f.argtypes)])
    out.append([rc, log(0).decode()])
print("RESULT" + json.dumps(out))
"""


def build(folder):
    out = os.path.join(str(folder), "launch_log.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-o", out, os.path.join(HERE, "launch_log.cpp")], check=True)
    return out


def launches(log, calls):
    """calls: (entry point, arguments, bytes of each kernel's first argument to look at).  For each: (return code, [(kernel, template arguments, grid, block, bytes)])."""
    env = {**os.environ, "LD_PRELOAD": log, "HIP_VISIBLE_DEVICES": "", "PYTHONPATH": os.path.dirname(HERE)}
    r = subprocess.run([sys.executable, "-c", CHILD, log], input=json.dumps(calls), env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    out = []
    for rc, text in json.loads(r.stdout.split("RESULT")[1]):
        made = []
        for line in text.splitlines():
            name, *numbers = line.split(" ")
            m = re.match(r"_ZN12_GLOBAL__N_1\d+([a-z_0-9]+_kernel)(?:I(.*)EE)?", name)
            n = [int(x) for x in numbers[:6]]
            args = re.findall(r"L(?:[a-z]|NS_\d+[A-Za-z]+E|N12_GLOBAL__N_1\d+[A-Za-z]+E)(\d+)E", (m.group(2) or "") + "E")
            made.append((m.group(1), tuple(int(x) for x in args), tuple(n[:3]), tuple(n[3:6]), bytes.fromhex(numbers[6])))
        out.append((rc, made))
    return out
