"""The host code of the expert-layer operators under a HIP runtime that computes nothing (fake_hip.cpp), in a process of its own: what their plans allocate,
what their calls launch, on a machine without a GPU.

    ask([{"op": "scaled", "M": 8, "N": 8, "K": 8, ...}, {"op": "route", "tokens": 4, ...}, ...]) -> one dict per question: status of the plan, description,
    workspace bytes, launches as [kernel, grid x, grid y] of one run (and of a gradient) on a stream of its own, and how many of them did not wait for the clearing
    of the plan's memory.  Operands lie at an address that nothing reads."""
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
BASE, STREAM = 1 << 36, 1 << 20         # STREAM: not the null stream


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
        fake.fake_take_overtaken()
        r["run"], r["launches"] = lib.hgemm_scaled_run(plan, *[BASE] * 5, BASE, BASE, STREAM), _launches(fake)
        r["overtaken"] = fake.fake_take_overtaken()
        lib.hgemm_scaled_destroy(plan)
    return r


def _route(fake, lib, experts, q):
    d = experts._Route(**{"groups": 1, "keep": 1, "align": 1, "factor": 1.0, **{n: q[n] for n, _ in experts._Route._fields_ if n in q}})
    plan = ctypes.c_void_p()
    r = {"plan": lib.hgemm_route_plan(ctypes.byref(plan), ctypes.byref(d))}
    if r["plan"] == 0:
        fake.fake_take_log()
        fake.fake_take_overtaken()
        r["run"], r["launches"] = lib.hgemm_route_run(plan, BASE, None, *[BASE] * 5, STREAM), _launches(fake)
        r["overtaken"] = fake.fake_take_overtaken()
        r["backward"], r["backward_launches"] = lib.hgemm_route_backward(plan, *[BASE] * 4, STREAM), _launches(fake)
        lib.hgemm_route_destroy(plan)
    return r


def _plan(fake, lib, experts, q):
    """A product of 16-bit floats (hgemm_plan_override)."""
    plan = ctypes.c_void_p()
    i64 = ctypes.c_int64
    r = {"plan": lib.hgemm_plan_override(ctypes.byref(plan), i64(q["M"]), i64(q["N"]), i64(q["K"]), None, q["spec"].encode())}
    if r["plan"] == 0:
        r["workspace"] = lib.hgemm_plan_workspace_bytes(plan)
        fake.fake_take_overtaken()
        r["run"] = lib.hgemm_run(plan, *[ctypes.c_void_p(BASE)] * 3, ctypes.c_void_p(STREAM))
        r["overtaken"] = fake.fake_take_overtaken()
        lib.hgemm_destroy(plan)
    return r


if __name__ == "__main__":
    fake_lib = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    fake_lib.fake_take_log.restype = ctypes.c_char_p
    fake_lib.fake_live_bytes.restype = ctypes.c_size_t
    from paper_2512_02551_amd import experts as experts_module
    hgemm_lib = ctypes.CDLL(LIB)
    experts_module.declare(hgemm_lib)
    hgemm_lib.hgemm_plan_workspace_bytes.restype = ctypes.c_size_t
    answers = [{"scaled": _scaled, "route": _route, "plan": _plan}[q["op"]](fake_lib, hgemm_lib, experts_module, q) for q in json.load(sys.stdin)]
    assert fake_lib.fake_live_bytes() == 0, "a plan's memory was not given back"
    print(json.dumps(answers))
