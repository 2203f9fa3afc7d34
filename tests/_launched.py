"""Which kernel a call launches first, without a GPU: in a process that sees no device every launch is refused, and the error
names the kernel. (Addresses are made up; where a device is visible all the same, no call is made.)"""
import ctypes
import json
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def launched(calls):
    """The names for a list of (function, arguments); an argument "@n" is the address n, a result >= 0 or a refusal by the
    checks comes back as it is."""
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", PYTHONPATH=ROOT)
    out = subprocess.run([sys.executable, "-m", "tests._launched"], input=json.dumps(calls), capture_output=True, text=True, env=env,
                         cwd=ROOT, timeout=120)
    assert out.returncode == 0, out.stderr
    return json.loads(out.stdout)


def _main():
    from paper_1712_04432_amd._abi import load
    lib = load()
    n = ctypes.c_int(0)
    lib.hipGetDeviceCount(ctypes.byref(n))
    assert n.value == 0, "a device is visible"
    names = []
    for name, args in json.load(sys.stdin):
        args = [ctypes.c_void_p(int(a[1:])) if isinstance(a, str) else a for a in args]
        code = getattr(lib, name)(*args)
        text = lib.imbd_last_error().decode()
        names.append(text.split(": launch failed")[0] if code == -3 and ": launch failed" in text else [code, text])
    json.dump(names, sys.stdout)


if __name__ == "__main__":
    _main()
