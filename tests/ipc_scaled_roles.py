"""The three processes of the attach test of 8-bit pools (tests/test_gpu_scaled_pools.py), run as `python tests/ipc_scaled_roles.py ROLE ...`:

  launcher  touches no GPU: starts the exporter, hands its handles to the importer, tells the exporter to leave, exits with the importer's status.
  exporter  allocates the two 8-bit pools, fills them with seeded experts and exports them.
  importer  builds a layer over the attached pools (the scales are its own) and checks a pass against 64 bits.
"""
import json
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
sys.path.insert(0, os.path.join(ROOT, "tests"))

SHAPE = dict(H=256, I=144, E=16, k=4, n_local=5, n_shared=1, seed=1)


def launcher():
    me = os.path.abspath(__file__)
    exp = subprocess.Popen([sys.executable, "-u", me, "exporter"], stdin=subprocess.PIPE, stdout=subprocess.PIPE, text=True)
    try:
        line = exp.stdout.readline()
        if not line.startswith("{"):
            print("launcher: exporter did not deliver handles:", line, flush=True)
            return 3
        return subprocess.run([sys.executable, "-u", me, "importer", line.strip()], timeout=100).returncode
    finally:
        try:
            exp.stdin.write("leave\n")
            exp.stdin.flush()
        except OSError:
            pass
        try:
            exp.wait(timeout=30)
        except subprocess.TimeoutExpired:
            exp.kill()


def exporter():
    import torch
    from paper_2510_02613_amd.layer import export_pool
    from test_gpu_scaled_layer import Layer
    L = Layer(**SHAPE)
    torch.cuda.synchronize()
    (h13, o13), (h2, o2) = export_pool(L.pools.w13), export_pool(L.pools.w2)
    print(json.dumps({"w13": [h13.hex(), o13], "w2": [h2.hex(), o2], "pid": os.getpid()}), flush=True)
    sys.stdin.readline()
    torch.cuda.synchronize()


def importer(arg):
    import torch
    from paper_2510_02613_amd.layer import AttachedPool
    from test_gpu_scaled_layer import Layer
    from test_gpu_scaled_pools import over_pools, same_as_plain
    h = json.loads(arg)
    assert h["pid"] != os.getpid()
    L = Layer(**SHAPE)                               # the same experts, slots and scales in memory of its own
    shapes = [tuple(t.shape) for t in (L.pools.w13, L.pools.w2)]
    p13, p2 = (AttachedPool(bytes.fromhex(h[name][0]), h[name][1], shape[0], shape[1:], torch.float8_e4m3fn) for name, shape in zip(("w13", "w2"), shapes))
    layer = over_pools(L, p13, p2, L.pools.w13_scale, L.pools.w2_scale)
    assert layer.w13.data_ptr() == p13.ptr and layer.w2.data_ptr() == p2.ptr
    same_as_plain(L, layer)
    layer.close()
    L.close()
    p13.close()
    p2.close()
    print("importer: passes on attached 8-bit pools OK", flush=True)


if __name__ == "__main__":
    role = sys.argv[1]
    if role == "launcher":
        sys.exit(launcher())
    if role == "exporter":
        exporter()
    elif role == "importer":
        importer(sys.argv[2])
    else:
        sys.exit(f"unknown role {role}")
