"""The host code of the expert-layer operators under a HIP runtime that computes nothing (fake_hip.cpp), in a process of its own: what their plans allocate,
what their calls launch, on a machine without a GPU.

    ask([{"op": "scaled", "M": 8, "N": 8, "K": 8, ...}, {"op": "route", "tokens": 4, ...}, ...]) -> one dict per question: status of the plan, description,
    workspace bytes, launches as [kernel, grid x, grid y] of one run (and of a gradient).  Operands lie at an address that nothing reads."""
import ctypes
import json
import os
import re
import subprocess
import sys
import tempfile

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.dirname(HERE))
LIB = os.path.join(os.path.dirname(HERE), "paper_2512_02551_amd", "libhgemm.so")
BASE = 1 << 36


def ask(questions):
    with tempfile.TemporaryDirectory() as tmp:
        so = os.path.join(tmp, "libfake_hip.so")
        subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-I/opt/rocm/include", os.path.join(HERE, "fake_hip.cpp"), "-o", so], check=True)
        res = subprocess.run([sys.executable, os.path.abspath(__file__), so], input=json.dumps(questions), stdout=subprocess.PIPE, text=True, check=True)
    return json.loads(res.stdout)


def _launches(fake):
    found = []
    for line in fake.fake_take_log().decode().splitlines():
        if line.startswith("launch "):
            name, x, y = line.split()[1:4]
            found.append([re.search(r"((?:scaled|route|place|quantise|combine)[a-z0-9_]*?_kernel)", name)[1], int(x), int(y)])
    return found


def _scaled(fake, lib, experts, q):
    d = experts._Scaled(**{"b_block_rows": 128, **{n: q[n] for n, _ in experts._Scaled._fields_ if n in q}})
    plan = ctypes.c_void_p()
    args = [ctypes.byref(plan), q["M"], q["N"], q["K"], ctypes.byref(d)]
    r = {"plan": lib.hgemm_scaled_plan_override(*args, q["spec"].encode()) if "spec" in q else lib.hgemm_scaled_plan(*args)}
    if r["plan"] == 0:
        text = ctypes.create_string_buffer(256)
        assert lib.hgemm_scaled_describe(plan, text, 256) == 0
        fake.fake_take_log()
        r["describe"], r["workspace"] = text.value.decode(), lib.hgemm_scaled_workspace_bytes(plan)
        r["run"], r["launches"] = lib.hgemm_scaled_run(plan, *[BASE] * 5, BASE, BASE, None), _launches(fake)
        lib.hgemm_scaled_destroy(plan)
    return r


def _route(fake, lib, experts, q):
    d = experts._Route(**{"groups": 1, "keep": 1, "align": 1, "factor": 1.0, **{n: q[n] for n, _ in experts._Route._fields_ if n in q}})
    plan = ctypes.c_void_p()
    r = {"plan": lib.hgemm_route_plan(ctypes.byref(plan), ctypes.byref(d))}
    if r["plan"] == 0:
        fake.fake_take_log()
        r["run"], r["launches"] = lib.hgemm_route_run(plan, BASE, None, *[BASE] * 5, None), _launches(fake)
        r["backward"], r["backward_launches"] = lib.hgemm_route_backward(plan, *[BASE] * 4, None), _launches(fake)
        lib.hgemm_route_destroy(plan)
    return r


if __name__ == "__main__":
    fake_lib = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    fake_lib.fake_take_log.restype = ctypes.c_char_p
    fake_lib.fake_live_bytes.restype = ctypes.c_size_t
    from paper_2512_02551_amd import experts as experts_module
    hgemm_lib = ctypes.CDLL(LIB)
    experts_module.declare(hgemm_lib)
    answers = [{"scaled": _scaled, "route": _route}[q["op"]](fake_lib, hgemm_lib, experts_module, q) for q in json.load(sys.stdin)]
    assert fake_lib.fake_live_bytes() == 0, "a plan's memory was not given back"
    print(json.dumps(answers))
