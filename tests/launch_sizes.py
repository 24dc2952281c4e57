"""What calls launch, on a stand-in for the HIP runtime that refuses what a GPU's launch
does (launch_sizes.cpp): nothing is executed and no pointer is used.

launches() runs calls (name, arguments: numbers, None, or a list for a structure of
pointers) in a process of its own and returns each one's status and launches, as (kernel,
workgroups in x)."""
import json
import os
import subprocess
import sys

from fake_hip import HERE, LIB


def build(folder) -> str:
    so = os.path.join(str(folder), "liblaunch_sizes.so")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__",
                    "-I/opt/rocm/include", os.path.join(HERE, "launch_sizes.cpp"), "-o", so],
                   check=True)
    return so


def launches(so: str, calls: list) -> list:
    out = subprocess.run([sys.executable, os.path.abspath(__file__), so, LIB, json.dumps(calls)],
                         check=True, capture_output=True, text=True, timeout=120).stdout
    return json.loads(out)


def _run(so, lib, calls):
    import ctypes
    fake = ctypes.CDLL(so, mode=ctypes.RTLD_GLOBAL)
    fake.fake_log.restype = ctypes.c_char_p
    L = ctypes.CDLL(lib)
    done, results = 0, []

    def plain(a):
        if isinstance(a, list):
            return ctypes.byref((ctypes.c_void_p * len(a))(*a))
        if isinstance(a, float):
            return ctypes.c_float(a)
        return ctypes.c_int64(a) if isinstance(a, int) and a >> 31 else a

    for name, args in calls:
        status = getattr(L, name)(*[plain(a) for a in args])
        log = fake.fake_log().decode()
        results.append((status, [(k, int(n)) for k, n in
                                 (line.rsplit(" ", 1) for line in log[done:].splitlines())]))
        done = len(log)
    print(json.dumps(results))


if __name__ == "__main__":
    _run(sys.argv[1], sys.argv[2], json.loads(sys.argv[3]))
