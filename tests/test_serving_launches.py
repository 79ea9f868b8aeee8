"""What the served decoding step launches, without a GPU: the library on top of a recorder in the place of the HIP runtime (launch_recorder.cpp), in a process of
its own."""
import ctypes
import json
import os
import subprocess
import sys
import types

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
A = 1 << 40


def record(calls, tmp_path):
    """(return code, launches) of each call: {"entry", "desc", and for w4 "tokens"; "device", "fail"}; a launch is (kernel, grid, block, dynamic LDS, cap on it)."""
    lib = os.path.join(str(tmp_path), "launch_recorder.so")
    if not os.path.exists(lib):
        subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", os.path.join(HERE, "launch_recorder.cpp"), "-o", lib], check=True)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), lib], input=json.dumps(calls), capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr[-2000:]
    return [(rc, [tuple(l) for l in launches]) for rc, launches in json.loads(r.stdout)]


def _main(recorder):
    rec = ctypes.CDLL(recorder, mode=ctypes.RTLD_GLOBAL)      # before the library: its symbols resolve to these first
    rec.rec_name.restype = ctypes.c_char_p
    sys.modules["torch"] = types.ModuleType("torch")          # no other HIP runtime in this process
    sys.path.insert(0, os.path.dirname(HERE))
    from paper_2505_19342_amd import binding as B
    lib = B.load(build_if_missing=False)
    out = []
    for c in json.load(sys.stdin):
        rec.rec_reset(c.get("device", 0), int(c.get("fail", False)))
        if c["entry"] == "w4":
            d = B.w4_desc(*c["desc"])
            rc = lib.astra_w4_linear(ctypes.byref(d), A, c["tokens"], A, A, None, None, A, None)
        else:
            d = B.cache_desc(**c["desc"])
            if c["entry"] == "append":
                rc = lib.astra_cache_append(ctypes.byref(d), A, A, A, None, A, A, A, A, A, A, A, A, None)
            else:
                n = lib.astra_cache_attention_workspace_bytes(ctypes.byref(d))
                rc = lib.astra_cache_attention(ctypes.byref(d), A, A, A, A, A, A, A, A, None, None, A, None, A, n, None)
        launches = []
        for i in range(rec.rec_count()):
            grid, block = (ctypes.c_uint32 * 3)(), (ctypes.c_uint32 * 3)()
            lds, cap = ctypes.c_size_t(), ctypes.c_size_t()
            rec.rec_shape(i, grid, block, ctypes.byref(lds), ctypes.byref(cap))
            name = rec.rec_name(i).decode().replace("void ", "").replace("astra::", "").split("(")[0]
            launches.append((name.replace("unsigned short", "bf16"), list(grid), list(block), lds.value, cap.value))
        out.append((rc, launches))
    json.dump(out, sys.stdout)


W4 = [  # element type, tokens, in, out -> kernel, grid
    ("bf16", 1, 4096, 4096, "w4_kernel<bf16, 2, 7, 2>", (256, 1)), ("bf16", 2, 4096, 4097, "w4_kernel<bf16, 2, 7, 2>", (257, 1)),
    ("bf16", 3, 4096, 1, "w4_kernel<bf16, 8, 7, 2>", (1, 1)), ("bf16", 8, 128, 100, "w4_kernel<bf16, 8, 7, 2>", (7, 1)),
    ("bf16", 9, 14336, 4096, "w4_kernel<bf16, 16, 7, 2>", (256, 1)), ("bf16", 16, 4096, 4096, "w4_kernel<bf16, 16, 7, 2>", (256, 1)),
    ("bf16", 17, 4096, 4096, "w4_wide_kernel<2, 2, 4, 1, 2, 7>", (128, 1)), ("bf16", 33, 4096, 4096, "w4_wide_kernel<2, 2, 4, 1, 2, 7>", (128, 2)),
    ("bf16", 20, 256, 24449, "w4_wide_kernel<2, 4, 2, 2, 1, 7>", (192, 1)), ("bf16", 20, 256, 24448, "w4_wide_kernel<2, 2, 4, 1, 1, 7>", (764, 1)),
    ("bf16", 64, 256, 24449, "w4_wide_kernel<4, 4, 2, 2, 1, 7>", (192, 1)), ("bf16", 65, 256, 12288, "w4_wide_kernel<4, 4, 2, 2, 1, 7>", (96, 2)),
    ("bf16", 64, 256, 12288, "w4_wide_kernel<2, 4, 2, 2, 1, 7>", (96, 2)), ("bf16", 1 << 19, 128, 16, "w4_wide_kernel<4, 4, 2, 2, 1, 7>", (1, 8192)),
    ("bf16", 65, 4096, 4096, "w4_wide_kernel<2, 2, 4, 1, 1, 7>", (128, 3)),
    ("f32", 1, 4096, 4096, "w4_kernel<float, 2, 7, 1>", (256, 1)), ("f32", 16, 4096, 4096, "w4_kernel<float, 16, 7, 1>", (256, 1)),
    ("f32", 17, 4096, 4096, "w4_kernel<float, 16, 7, 1>", (256, 2)), ("f32", 1 << 19, 128, 16, "w4_kernel<float, 16, 7, 1>", (1, 32768)),
]


def test_products(tmp_path):
    results = record([dict(entry="w4", desc=(dt, k, n, 128), tokens=t) for dt, t, k, n, _, _ in W4], tmp_path)
    for (dt, t, k, n, name, grid), (rc, launches) in zip(W4, results):
        assert rc == 0 and [(l[0], tuple(l[1])) for l in launches] == [(name, grid + (1,))], (dt, t, k, n, launches)


CACHE = dict(n_q_heads=32, n_kv_heads=8, head_dim=128, page_size=64, n_pages=1000)


def cache(dtype="bf16", **change):
    return {"dtype": dtype, **CACHE, **change}


def test_appends(tmp_path):
    """One launch: workgroups of a wavefront where sequences have few rows, of four where they have 16 or more on average."""
    cases = [(cache(n_seqs=1, n_tokens=1, max_pages=10), "cache_append_kernel<bf16, 128, 64>", 16 + 2), (cache(n_seqs=64, n_tokens=64, max_pages=10), "cache_append_kernel<bf16, 128, 64>", 1024 + 128),
             (cache(n_seqs=64, n_tokens=2047, max_pages=10, dtype="f32"), "cache_append_kernel<float, 128, 256>", 128 * 16 + 2047 * 8 // 16 + 1),
             (cache(n_seqs=4, n_tokens=8192, max_pages=100, head_dim=64), "cache_append_kernel<bf16, 64, 256>", 128 * 16 + 2048)]
    for (d, name, blocks), (rc, launches) in zip(cases, record([dict(entry="append", desc=c[0]) for c in cases], tmp_path)):
        assert rc == 0 and [(l[0], l[1][0]) for l in launches] == [(name, blocks)], (d, launches)


def test_attention_cut_or_whole(tmp_path):
    """Whole sequences and one launch where none can be long; equal shares and a second launch otherwise, with no more workgroups than the units hold at a time."""
    def whole(t, dh, nt, wide=True):
        return [f"cache_attn_kernel<{dh}, {t}, {nt}, false, {str(wide).lower()}>"]

    def cut(t, dh, nt):
        return [f"cache_attn_kernel<{dh}, {t}, {nt}, true, false>", f"cache_attn_join_kernel<{dh}, {t}, {nt}>"]
    cases = [(cache(n_seqs=1, n_tokens=1, max_pages=12), whole("bf16", 128, 1), 8), (cache(n_seqs=32, n_tokens=32, max_pages=40), whole("bf16", 128, 1), 320),
             (cache(n_seqs=33, n_tokens=33, max_pages=40), whole("bf16", 128, 1, False), 328), (cache(n_seqs=1, n_tokens=1, max_pages=12, dtype="f32", head_dim=256), whole("float", 256, 1, False), 8), (cache(n_seqs=1, n_tokens=1, max_pages=13), cut("bf16", 128, 1), 13 * 8),
             (cache(n_seqs=64, n_tokens=64, max_pages=64), whole("bf16", 128, 1, False), 640), (cache(n_seqs=64, n_tokens=64, max_pages=65), cut("bf16", 128, 1), 768),
             (cache(n_seqs=2, n_tokens=512, max_pages=64), whole("bf16", 128, 2, False), 528), (cache(n_seqs=2, n_tokens=512, max_pages=65, dtype="f32"), cut("float", 128, 1), 512),
             (cache(n_seqs=2, n_tokens=512, max_pages=65, head_dim=256), cut("bf16", 256, 1), 512), (cache(n_seqs=2, n_tokens=512, max_pages=65, head_dim=64), cut("bf16", 64, 2), 768)]
    for (d, names, wgs), (rc, launches) in zip(cases, record([dict(entry="attend", desc=c[0]) for c in cases], tmp_path)):
        assert rc == 0 and [l[0] for l in launches] == names and launches[0][1][0] == wgs, (d, launches)
        if len(names) > 1:
            joins, rows = wgs, d["n_tokens"] * d["n_q_heads"] // d["n_kv_heads"]
            assert launches[1][1][:2] == ([8, 4] if d["n_seqs"] == 1 else [joins, min(rows, 16384 // joins, 16 * int(names[1][-2]))]), (d, launches)


def test_the_cap_on_dynamic_lds_is_raised_on_every_device_and_a_refusal_is_an_error(tmp_path):
    calls = [dict(entry="w4", desc=(dt, 14336, 24500, g), tokens=t, device=d, fail=f)
             for f in (True, False) for d in (0, 1, 70, 0) for g in (32, 64, 128) for dt, t in (("bf16", 1), ("bf16", 16), ("f32", 1), ("f32", 8), ("f32", 16), ("bf16", 20), ("bf16", 64))]
    large = 0
    for c, (rc, launches) in zip(calls, record(calls, tmp_path)):
        if c["fail"] and rc:
            large += 1
            assert not launches
            continue
        assert rc == 0 and len(launches) == 1, (c, rc)
        name, _, _, lds, cap = launches[0]
        assert lds <= (cap or 64 * 1024) and lds <= 160 * 1024, (c, launches)
        assert not c["fail"] or lds <= 64 * 1024
    assert large


def test_what_passes_a_limit_is_refused(tmp_path):
    UNSUPPORTED, SHAPE = -5, -2
    big = cache(n_seqs=4, n_tokens=1 << 24, max_pages=1 << 19)
    calls = [(dict(entry="w4", desc=("bf16", 512, 100, 64, "bf16", (1 << 25) + 8), tokens=3), UNSUPPORTED), (dict(entry="w4", desc=("bf16", 512, 100, 64), tokens=(1 << 19) + 1), SHAPE),
             (dict(entry="w4", desc=("bf16", 512, (1 << 24) + 1, 64), tokens=3), UNSUPPORTED), (dict(entry="append", desc=dict(big, n_tokens=(1 << 24) + 1)), UNSUPPORTED),
             (dict(entry="attend", desc=big), UNSUPPORTED),                                                   # 2^19 row blocks of 2^20 tiles each
             (dict(entry="append", desc=dict(big, n_q_heads=4096)), UNSUPPORTED),                             # 2^34 groups of query heads
             (dict(entry="attend", desc=dict(big, n_q_heads=4096, n_kv_heads=1)), UNSUPPORTED),               # 2^36 rows of queries
             (dict(entry="attend", desc=dict(big, max_pages=1, n_q_heads=64, n_kv_heads=64)), UNSUPPORTED)]   # 2^25 row blocks
    for (c, want), (rc, launches) in zip(calls, record([c for c, _ in calls], tmp_path)):
        assert rc == want and not launches, (c, rc)


if __name__ == "__main__":
    _main(sys.argv[1])
