"""Which kernels an attention call would launch, found out without a GPU: as launch_record.py, whose stand-in for the HIP runtime it
compiles, for the calls of attention_sizes.py."""
import ctypes as C
import json
import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))


def record(calls, folder):
    """calls: [["forward" or "backward", *AttentionSpec's fields up to dtype], ["paged", requests, longest, heads, key heads, elements, page, dtype]].
    Returns [(status, [kernel, ...]), ...]."""
    shim = os.path.join(str(folder), "launch_record.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-Wall", "-o", shim, os.path.join(HERE, "launch_record.c")], check=True)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), shim, os.path.dirname(HERE)], input=json.dumps(calls), capture_output=True,
                       text=True, timeout=600)
    assert r.returncode == 0, r.stderr
    return json.loads(r.stdout.splitlines()[-1])


def _make(B, L, what, *args):
    from paper_1804_04512_amd.workloads import AttentionSpec, CacheSpec
    p, ws, room = [C.c_void_p((k + 2) << 40) for k in range(12)], C.c_void_p(1 << 20), 1 << 62   # made-up addresses, far apart
    if what == "paged":
        requests, longest, heads, kv_heads, dim, page, dtype = args
        d = C.byref(B.cache_desc(CacheSpec(requests, heads, kv_heads, dim, 1 << 16, page, -(-longest // page), dtype)))
        return L.dll_paged_attention(d, *p[:5], 1.0, p[5], p[6], ws, room, None)
    d = C.byref(B.attention_desc(AttentionSpec(*args)))
    if what == "forward":
        return L.dll_attention_fwd(d, *p[:5], 1.0, p[5], p[6], ws, room, None)
    return L.dll_attention_bwd(d, *p[:5], 1.0, *p[5:11], ws, room, None)


def _main():
    shim = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)   # before anything that brings the runtime along
    sys.path.insert(0, sys.argv[2])
    from paper_1804_04512_amd import binding as B
    L = B.lib()
    text = C.create_string_buffer(1 << 18)
    shim.take_launches.argtypes = [C.c_char_p, C.c_size_t]
    out = []
    for call in json.load(sys.stdin):
        status = _make(B, L, *call)
        shim.take_launches(text, 1 << 18)
        out.append([status, [line.rsplit(" ", 4)[0] for line in text.value.decode().splitlines()]])
    print(json.dumps(out))


if __name__ == "__main__":
    _main()
