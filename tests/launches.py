"""The kernels that a call would launch, without a GPU: a process of its own loads tests/launch_recorder.cpp in the HIP runtime's place.

launches([("gp_embedding", {...}), ...]) makes the calls with these keyword arguments and returns, for each, what came of it:
dict(status, launches), a launch being dict(kernel, grid, block, lds, lds_asked).  An argument of no_memory=True lets the library's own
allocations fail during the call, with every kernel timed (gp_profile_enable), so that there are some.
"""
from __future__ import annotations

import atexit
import functools
import json
import os
import shutil
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))


@functools.lru_cache(maxsize=None)
def _recorder():
    folder = tempfile.mkdtemp(prefix="launches")
    atexit.register(shutil.rmtree, folder, ignore_errors=True)
    path = os.path.join(folder, "recorder.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-fvisibility=default", os.path.join(HERE, "launch_recorder.cpp"), "-o", path], check=True)
    return path


def launches(calls):
    done = subprocess.run([sys.executable, os.path.abspath(__file__), _recorder()], input=json.dumps(calls), capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, f"the process ended with {done.returncode}: {done.stderr[-2000:]}"
    return json.loads(done.stdout)


def _child(recorder_path, calls):
    import ctypes
    sys.modules["torch"] = None  # (it brings a HIP runtime of its own)
    recorder = ctypes.CDLL(recorder_path, mode=ctypes.RTLD_GLOBAL)
    recorder.recorder_count.restype = ctypes.c_int64
    recorder.recorder_name.restype = ctypes.c_char_p
    recorder.recorder_name.argtypes = [ctypes.c_int64]
    recorder.recorder_sizes.argtypes = [ctypes.c_int64, ctypes.POINTER(ctypes.c_uint64)]
    sys.path.insert(0, os.path.dirname(HERE))
    import paper_2207_12000_amd as gp
    results = []
    for name, kw in calls:
        kw = dict(kw)
        no_memory = kw.pop("no_memory", False)
        recorder.recorder_clear()
        status = gp.GP_OK
        if no_memory:
            gp.gp_profile_enable(True)
            recorder.recorder_no_memory(1)
        try:
            getattr(gp, name)(**kw)
        except gp.GpError as e:
            status = e.status
        recorder.recorder_no_memory(0)
        seen = []
        for i in range(recorder.recorder_count()):
            v = (ctypes.c_uint64 * 8)()
            recorder.recorder_sizes(i, v)
            seen.append(dict(kernel=recorder.recorder_name(i).decode(), grid=list(v[0:3]), block=list(v[3:6]), lds=v[6], lds_asked=v[7]))
        results.append(dict(status=status, launches=seen))
    return results


if __name__ == "__main__":
    sys.stdout.write(json.dumps(_child(sys.argv[1], json.loads(sys.stdin.read()))))
