"""Which kernels the entry points launch, without a GPU: the library in a process of its own on a runtime that writes launches down (host_runtime.cpp).

    runtime(calls) -> for each (entry point, its arguments) the status and what was launched and raised

An argument that is a float is a float, any other an integer or an address; addresses are not followed."""
import collections
import json
import os
import subprocess
import sys

from paper_2502_08145_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
Launch = collections.namedtuple("Launch", "kernel workgroups threads lds")   # kernel: its mangled name
Answer = collections.namedtuple("Answer", "status launches limits")   # limits: (kernel, bytes of LDS)

_CHILD = """
import ctypes, json, sys
fake = ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
fake.host_runtime_log.restype = ctypes.c_char_p
for name, args in json.load(sys.stdin):
    fake.host_runtime_clear()
    status = getattr(lib, name)(*[ctypes.c_float(a) if isinstance(a, float) else ctypes.c_int64(a) for a in args])
    print(json.dumps([status, fake.host_runtime_log().decode()]))
"""


def build_runtime(folder) -> str:
    so = os.path.join(str(folder), "host_runtime.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-shared", "-fPIC", os.path.join(HERE, "host_runtime.cpp"), "-o", so], check=True)
    return so


def run(so, calls):
    out = subprocess.run([sys.executable, "-c", _CHILD, so, build.LIB], input=json.dumps(list(calls)), capture_output=True, text=True, check=True, timeout=100).stdout
    answers = []
    for line in out.splitlines():
        status, log = json.loads(line)
        launches, limits = [], []
        for what, kernel, workgroups, threads, lds in (entry.split() for entry in log.splitlines()):
            if what == "launch":
                launches.append(Launch(kernel, int(workgroups), int(threads), int(lds)))
            else:
                limits.append((kernel, int(lds)))
        answers.append(Answer(status, launches, limits))
    return answers


def readable(kernels):
    """{mangled name: name with its template arguments}"""
    kernels = sorted(set(kernels))
    out = subprocess.run(["c++filt"], input="\n".join(kernels), capture_output=True, text=True, check=True).stdout.splitlines()
    return {k: line.split("(")[0].replace("void ", "").replace("axonn::", "") for k, line in zip(kernels, out)}


def kernels_of_the_library(so):
    """The mangled names of all kernels, as the library registers them"""
    code = "import ctypes, sys; f = ctypes.CDLL(sys.argv[1], ctypes.RTLD_GLOBAL); ctypes.CDLL(sys.argv[2]); f.host_runtime_kernels.restype = ctypes.c_char_p; print(f.host_runtime_kernels().decode())"
    return subprocess.run([sys.executable, "-c", code, so, build.LIB], capture_output=True, text=True, check=True, timeout=100).stdout.split()
