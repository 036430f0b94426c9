"""Which kernels the calls on dense matrices launch, found without a GPU, as routes.py does for the layer's:

    routes([dict(fn="orthogonalize", batch=3, rows=8, cols=16), ...], recorder_path)

gives for every call (status, [(kernel, grid, threads, LDS bytes), ...], workspace bytes).  A call is a dict of
  fn         "orthogonalize", "muon", "quantize" or "linear"
  batch, rows, cols, dtype, schedule (default: five steps of the quintic)     the first two
  rows, cols, dtype                                                          quantize
  batch, n_in, n_out, x_dtype, y_dtype, w (offset of the weights, bytes)     linear
"""
import ctypes as C
import json
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
LIBRARY = os.path.join(os.path.dirname(HERE), "paper_2509_07103_amd", "liblmkan.so")
QUINTIC = [[3.4445, -4.7750, 2.0315]] * 5


def routes(calls, recorder_path, library=LIBRARY):
    got = subprocess.run([sys.executable, os.path.abspath(__file__), recorder_path, library], input=json.dumps(calls),
                         capture_output=True, text=True)
    assert got.returncode == 0, got.stderr
    return [(status, [tuple(launch) for launch in launches], need) for status, launches, need in json.loads(got.stdout)]


class _Matrices(C.Structure):
    _fields_ = [("batch", C.c_int64), ("rows", C.c_int32), ("cols", C.c_int32), ("dtype", C.c_int32), ("eps", C.c_float)]


class _Muon(C.Structure):
    _fields_ = [(f, C.c_float) for f in ("lr", "momentum", "weight_decay", "scale")] + [("nesterov", C.c_int32)]


class _Linear(C.Structure):
    _fields_ = [(f, C.c_int32) for f in ("n_in", "n_out", "x_dtype", "y_dtype", "flags")]


def _main():
    rec = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
    lib = C.CDLL(sys.argv[2])
    rec.recorder_text.restype = C.c_char_p
    lib.lmkan_orthogonalize_workspace_bytes.restype = lib.lmkan_linear_i8_workspace_bytes.restype = C.c_size_t
    at = [C.c_void_p((i + 1) << 40) for i in range(8)]
    out = []
    for c in json.load(sys.stdin):
        rec.recorder_clear()
        need = 0
        if c["fn"] == "quantize":
            status = lib.lmkan_quantize_rows(C.c_int64(c["rows"]), c["cols"], c.get("dtype", 0), 0, at[0], at[1], at[2], None)
        elif c["fn"] == "linear":
            d = _Linear(c["n_in"], c["n_out"], c.get("x_dtype", 0), c.get("y_dtype", 0), 0)
            need = lib.lmkan_linear_i8_workspace_bytes(C.byref(d), C.c_int64(c["batch"]))
            status = lib.lmkan_linear_i8(C.byref(d), C.c_int64(c["batch"]), at[0], C.c_void_p(at[1].value + c.get("w", 0)), at[2], None,
                                         C.c_float(0.0), at[3], at[4], C.c_size_t(need), None)
        else:
            d = _Matrices(c["batch"], c["rows"], c["cols"], c.get("dtype", 0), 1e-7)
            flat = [v for row in c.get("schedule", QUINTIC) for v in row]
            schedule = (C.c_float * max(1, len(flat)))(*flat)
            need = lib.lmkan_orthogonalize_workspace_bytes(C.byref(d))
            rest = (len(flat) // 3, schedule), (at[3], C.c_size_t(need), None)
            if c["fn"] == "muon":
                m = _Muon(0.02, 0.95, 0.0, 1.0, 1)
                status = lib.lmkan_muon_step(C.byref(d), C.byref(m), *rest[0], at[0], at[1], at[2], *rest[1])
            else:
                status = lib.lmkan_orthogonalize(C.byref(d), *rest[0], at[0], at[1], *rest[1])
        launches = []
        for line in rec.recorder_text().decode().splitlines():
            name, grid, threads, lds = line.split("\t")
            launches.append((name, [int(v) for v in grid.split(",")], int(threads), int(lds)))
        out.append((status, launches, need))
    json.dump(out, sys.stdout)


if __name__ == "__main__":
    _main()
