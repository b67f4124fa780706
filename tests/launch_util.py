"""Which kernels a call launches, asked of the built library without a GPU: the library is loaded behind a stand-in for the HIP runtime
(host_launches/hip_stand_in.cpp) in a process of its own, and called with addresses that nobody follows."""
import ctypes
import json
import os
import shutil
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2401_11469_amd", "libzr.so")
STAND_IN = os.path.join(ROOT, "tests", "host_launches", "hip_stand_in.cpp")


def launches(tmp_path, calls):
    """calls: dicts of the arguments of zr_resized_linear_act_fwd that matter (M, K, N, n_keep or None, mode_k, kn, and `scratch`: whether
    there is a workspace).  For each a list of (demangled kernel, workgroups)."""
    shim = str(tmp_path / "hip_stand_in.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", STAND_IN, "-o", shim], check=True)
    env = {k: v for k, v in os.environ.items() if not k.startswith("ZR_")}
    run = subprocess.run([sys.executable, os.path.abspath(__file__), shim], input=json.dumps(calls), stdout=subprocess.PIPE, stderr=subprocess.PIPE,
                         text=True, env=env, timeout=120)
    assert run.returncode == 0, run.stderr[-2000:]
    text = run.stdout
    filt = shutil.which("llvm-cxxfilt") or shutil.which("c++filt")
    if filt:
        text = subprocess.run([filt], input=text, stdout=subprocess.PIPE, text=True, check=True).stdout
    out = []
    for line in text.splitlines():
        if line == "call":
            out.append([])
        else:
            name, groups = line.rsplit(" ", 1)
            out[-1].append((name.replace("zr::(anonymous namespace)::", "").replace("void ", ""), int(groups)))
    return out


def _main():
    shim = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    zr = ctypes.CDLL(LIB)
    vp, i64, i32, n, f64, size = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_int, ctypes.c_double, ctypes.c_size_t
    f = zr.zr_resized_linear_act_fwd
    f.argtypes = [vp, i64, vp, i64, vp, i64, i32, i32, i32, vp, i32, n, n, n, vp, n, vp, i64, f64, vp, vp, i64, vp, i64, vp, size, vp]
    space = zr.zr_act_fwd_workspace_bytes
    space.argtypes, space.restype = [i32, i32, i32, i32, n, n], size
    shim.launches_taken.restype, shim.launches_taken.argtypes = size, [ctypes.c_char_p, size]
    text = ctypes.create_string_buffer(1 << 16)
    at = lambda i: i << 40          # noqa: E731
    for c in json.loads(sys.stdin.read()):
        M, K, N, keep, mode_k, kn = c["M"], c["K"], c["N"], c["n_keep"], c["mode_k"], c["kn"]
        mode, layout, dtype = (1 if mode_k else 0), (0 if kn else 1), 1
        ws = space(M, K, N, keep or (K if mode_k else N), mode, dtype) if c["scratch"] else 0
        st = f(at(1), K, at(2), N if kn else K, at(3), N, M, K, N, at(4) if keep else None, keep or 0, mode, layout, dtype, None, 4, None, 0, 0.0, None,
               None, 0, None, 0, at(5) if ws else None, ws, None)
        assert st == 0, (st, c)
        assert shim.launches_taken(text, len(text)) <= len(text)
        print("call")
        print(text.value.decode(), end="")


if __name__ == "__main__":
    _main()
