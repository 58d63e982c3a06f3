"""Host side of the paged 8-bit KV cache without a GPU: sizes, refusals, and what is launched (a stand-in for the HIP runtime)."""
import ctypes as C
import os
import subprocess
import sys

import pytest

from paper_2512_15176_amd import binding

HERE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "hip_stub")
ROOT = os.path.dirname(os.path.dirname(HERE))

SCRIPT = """
import ctypes as C, mmap, sys
sys.path[:0] = [{root!r}, {here!r}]
stub = C.CDLL({lib!r}, mode=C.RTLD_GLOBAL)
stub.stub_launch.restype = C.c_char_p
from paper_2512_15176_amd import binding as B
lib = B.load_library()
mem = []
def buf(n):
    mem.append(mmap.mmap(-1, int(n)))
    return C.addressof(C.c_char.from_buffer(mem[-1]))
def make(**kw):
    p = B.kv8_params(**{{**dict(n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=64, max_batch=4, max_seq=1024, max_rows=2000), **kw}})
    s = B.Kv8Sizes()
    assert lib.deer_kv8_query_sizes(C.byref(p), C.byref(s)) == 0, lib.deer_kv8_last_error(None)
    ctx = C.c_void_p()
    assert lib.deer_kv8_init(C.byref(p), buf(s.cache), buf(s.workspace), C.byref(s), C.byref(ctx)) == 0
    return ctx
def launches():
    out = []
    for i in range(stub.stub_launches()):
        g = (C.c_uint32 * 3)()
        out.append((stub.stub_launch(i, g).decode(), tuple(g)))
    stub.stub_reset()
    return out
rows = buf(1 << 24)
ints = buf(1 << 16)
kv = make()
stub.stub_reset()
"""


def run(tmp_path, body):
    lib = os.path.join(str(tmp_path), "libkv8stub.so")
    subprocess.run(["gcc", "-O1", "-shared", "-fPIC", "-o", lib, os.path.join(HERE, "kv8_stub.c")], check=True)
    res = subprocess.run([sys.executable, "-c", SCRIPT.format(root=ROOT, here=HERE, lib=lib) + body], capture_output=True, text=True, timeout=120, cwd=ROOT)
    assert res.returncode == 0, res.stdout + res.stderr
    return res.stdout


def _sizes(**kw):
    p = binding.kv8_params(**{**dict(n_layers=36, n_q_heads=32, n_kv_heads=8, head_dim=128, max_batch=16, max_seq=32768, max_rows=512), **kw})
    s = binding.Kv8Sizes()
    return binding.load_library().deer_kv8_query_sizes(C.byref(p), C.byref(s)), s


def test_sizes_are_half_of_bf16():
    rc, s = _sizes()
    pool = 36 * 16 * 32768 * 8 * 128 * 2
    assert rc == 0 and pool < s.cache < 1.02 * pool
    rc, t = _sizes(n_pages=4096)
    assert rc == 0 and t.cache < 0.6 * s.cache and t.workspace == s.workspace


@pytest.mark.parametrize("bad", [dict(n_layers=0), dict(head_dim=96), dict(n_q_heads=12), dict(n_kv_heads=0), dict(n_q_heads=1024), dict(max_batch=0),
                                 dict(max_batch=1025), dict(max_seq=100), dict(max_seq=0), dict(max_seq=(1 << 20) + 64), dict(n_pages=-1),
                                 dict(n_pages=(1 << 24) + 1), dict(max_rows=0), dict(max_rows=(1 << 20) + 1)])
def test_shapes_are_checked(bad):
    rc, _ = _sizes(**bad)
    assert rc == -1 and binding.load_library().deer_kv8_last_error(None)


def test_versions_and_null_pointers():
    lib = binding.load_library()
    p, s, ctx = binding.kv8_params(1, 4, 2, 32, 1, 64), binding.Kv8Sizes(), C.c_void_p(1)
    p.struct_size += 4
    assert lib.deer_kv8_query_sizes(C.byref(p), C.byref(s)) == -5
    p.struct_size -= 4
    p.abi_version = 2
    assert lib.deer_kv8_query_sizes(C.byref(p), C.byref(s)) == -5
    p.abi_version = 1
    assert lib.deer_kv8_query_sizes(C.byref(p), None) == -1 and lib.deer_kv8_query_sizes(None, C.byref(s)) == -1
    assert lib.deer_kv8_query_sizes(C.byref(p), C.byref(s)) == 0
    assert lib.deer_kv8_init(C.byref(p), None, None, C.byref(s), C.byref(ctx)) == -1 and not ctx.value
    small = binding.Kv8Sizes(s.cache - 256, s.workspace)
    assert lib.deer_kv8_init(C.byref(p), 4096, 4096, C.byref(small), C.byref(ctx)) == -3 and not ctx.value
    assert lib.deer_kv8_init(C.byref(p), 4100, 4096, C.byref(s), C.byref(ctx)) == -1
    assert lib.deer_kv8_reserve(None, 1, None, None, 0, 0, 0) == -1 and lib.deer_kv8_destroy(None) == -1


def test_calls_refuse_what_the_kernels_cannot_take(tmp_path):
    run(tmp_path, """
I, S = -1, -2
assert lib.deer_kv8_append(kv, 0, rows, rows, 1, 128, 128, 0) == S and lib.deer_kv8_attend(kv, 0, rows, 1, 512, None, 0.0, rows, 512, 0) == S
R = lambda b, r, n, l, st=ints, nw=ints: lib.deer_kv8_reserve(kv, b, st, nw, r, n, l)
assert R(0, 1, 1, 1) == I and R(5, 1, 1, 1) == I and R(1, -1, 1, 1) == I and R(1, 2001, 1, 1) == I and R(1, 1, -1, 1) == I
assert R(1, 1, 1025, 1) == I and R(1, 1, 1, 1025) == I and R(1, 1, 1, -1) == I and R(1, 1, 1, 1, None) == I and R(1, 1, 1, 1, ints, ints + 2) == I
assert not launches()
assert R(4, 100, 40, 500) == 0
launches()
A = lambda layer=0, k=rows, v=rows, dt=1, ks=128, vs=128, n=100: lib.deer_kv8_append(kv, layer, k, v, dt, ks, vs, n)
for kw in (dict(layer=-1), dict(layer=2), dict(k=None), dict(v=rows + 8), dict(dt=2), dict(ks=127), dict(ks=132), dict(vs=120), dict(ks=0), dict(n=99), dict(ks=1 << 40)):
    assert A(**kw) == I, kw
Q = lambda layer=0, q=rows, dt=1, qs=512, lim=None, sc=0.0, o=rows, os=512, n=100: lib.deer_kv8_attend(kv, layer, q, dt, qs, lim, sc, o, os, n)
for kw in (dict(layer=2), dict(q=None), dict(o=rows + 4), dict(dt=5), dict(qs=511), dict(os=500), dict(lim=ints + 1), dict(sc=-1.0), dict(sc=float("nan")), dict(sc=float("inf")), dict(n=101)):
    assert Q(**kw) == I, kw
D = lambda layer=0, s=ints, p=ints, n=5, k=rows, v=rows, dt=1: lib.deer_kv8_read(kv, layer, s, p, n, k, v, dt)
for kw in (dict(layer=2), dict(s=None), dict(p=ints + 1), dict(n=-1), dict(k=None), dict(v=rows + 2), dict(dt=7)):
    assert D(**kw) == I, kw
assert not launches()
assert A(ks=136, vs=640) == 0 and A(dt=0, ks=132) == 0 and Q(sc=0.5) == 0 and Q(dt=0, lim=ints) == 0 and D(n=0) == 0 and D() == 0
names = [n for n, g in launches()]
assert [sum(w in n for n in names) for w in ("k_kv8_append", "k_kv8_attn", "k_kv8_read")] == [2, 2, 1]
stub.stub_fail(0, -1, -1)
assert R(4, 100, 40, 500) == -4 and b"planned" in lib.deer_kv8_last_error(kv)
assert lib.deer_kv8_destroy(kv) == 0
""")


def test_an_empty_pass_launches_only_its_tables(tmp_path):
    out = run(tmp_path, """
assert lib.deer_kv8_reserve(kv, 2, ints, ints, 0, 0, 1024) == 0
assert lib.deer_kv8_append(kv, 0, None, None, 1, 0, 0, 0) == 0 and lib.deer_kv8_attend(kv, 0, None, 1, 0, None, 0.0, None, 0, 0) == 0
print([n for n, g in launches()])
""")
    assert out.count("k_kv8") == 1 and "k_kv8_reserve" in out


def _engine_rc(**kw):
    import deer_inputs as di
    cfg = di.CONFIGS["tiny"]
    p = binding.init_params(cfg["target"], cfg["drafter"], 2, kw.pop("max_seq", 256), 8, 0, **kw)
    s = binding.Sizes()
    return binding.load_library().deer_query_sizes(C.byref(p), C.byref(s)), s, p


def test_an_engine_takes_the_format():
    rc, plain, p = _engine_rc()
    assert rc == 0
    p.struct_size = binding.InitParams.target_kv_format.offset          # a caller that does not know of it
    p.target_kv_format = 77
    s = binding.Sizes()
    assert binding.load_library().deer_query_sizes(C.byref(p), C.byref(s)) == 0 and s.kv[0] == plain.kv[0]
    rc, e8, _ = _engine_rc(kv_format=1)
    assert rc == 0 and e8.kv[1] == plain.kv[1] and e8.workspace == plain.workspace and e8.kv[0] != plain.kv[0]
    assert _engine_rc(kv_format=2)[0] == -1 and _engine_rc(kv_format=1, kv_pages=-1)[0] == -1
    assert _engine_rc(kv_format=1, max_seq=(1 << 20) + 64)[0] == -1


def test_an_engine_of_long_contexts_needs_half_the_memory():
    import deer_inputs as di
    cfg = di.CONFIGS["qwen3_8b_long_batch"]
    sizes = []
    for fmt in (0, 1):
        p = binding.init_params(cfg["target"], cfg["drafter"], 16, 32768 + 64, 32, 0, kv_format=fmt)
        s = binding.Sizes()
        assert binding.load_library().deer_query_sizes(C.byref(p), C.byref(s)) == 0
        sizes.append(s.kv[0])
    assert sizes[1] < 0.53 * sizes[0]


def test_an_engine_settles_pages_and_attends_in_8_bits(tmp_path):
    out = run(tmp_path, """
import deer_inputs as di
cfg = di.CONFIGS["tiny"]
t = di.scaled(cfg["target"], n_layers=5)
p = B.init_params(t, cfg["drafter"], 2, 256, 8, t.vocab - 1, kv_format=1, kv_pages=4)
s = B.query_sizes(p)
bufs = B.Buffers((C.c_void_p * 2)(*[buf(n) for n in s.weights]), (C.c_void_p * 2)(*[buf(n) for n in s.kv]), buf(s.workspace))
ctx = C.c_void_p()
assert lib.deer_init_models(C.byref(p), C.byref(bufs), C.byref(s), C.byref(ctx)) == 0
I32 = lambda v: (C.c_int32 * len(v))(*v)
pre = lambda lens: lib.deer_prefill(ctx, len(lens), I32([3] * sum(lens)), I32(lens))
assert pre([130, 130]) == -3                     # six pages of four
launches()
assert pre([130, 60]) == 0
names = [n for n, g in launches()]
count = lambda what: sum(what in n for n in names)
assert count("k_kv8_reserve") == 2 and count("k_kv8_prompt_pass") == 1
assert count("k_kv8_settle") == 5 and count("k_kv8_attn") == 4      # the last layer ends with its K and V rows
draft = (C.c_int32 * 64)()
assert lib.deer_draft_block(ctx, 8, C.c_float(0.0), 0, draft) == -3     # 129 + 8 and 59 + 8 tokens: 3 + 2 pages
assert lib.deer_draft_block(ctx, 5, C.c_float(0.0), 0, draft) == 0
launches()
assert lib.deer_verify_block(ctx, 5, C.c_float(0.0), draft) == 0
names = [n for n, g in launches()]
assert count("k_kv8_reserve") == 1 and count("k_kv8_settle") == 5 and count("k_kv8_attn") == 5      # 59 + 5 tokens: a page fills
assert lib.deer_debug_force_commit(ctx, (C.c_int32 * 2)(1, 1), (C.c_int32 * 2)(1, 1), 1) == 0
assert pre([130, 40]) == 0
assert lib.deer_draft_block(ctx, 5, C.c_float(0.0), 0, draft) == 0
launches()
assert lib.deer_verify_block(ctx, 5, C.c_float(0.0), draft) == 0
names = [n for n, g in launches()]
assert count("k_kv8_settle") == 0 and count("k_kv8_attn") == 5          # none does
assert not any("k_attn" in n for n in names)
print("done")
""")
    assert "done" in out


def test_a_long_pass_serves_one_layer_after_the_other(tmp_path):
    run(tmp_path, """
A = lambda layer: lib.deer_kv8_append(kv, layer, rows, rows, 1, 128, 128, 200)
Q = lambda layer: lib.deer_kv8_attend(kv, layer, rows, 1, 512, None, 0.0, rows, 512, 200)
R = lambda n: lib.deer_kv8_reserve(kv, 4, ints, ints, 200, n, 500)
assert R(65) == 0 and Q(0) == -2 and A(0) == 0 and Q(0) == 0 and Q(0) == 0 and A(0) == -2 and Q(1) == -2
assert A(1) == 0 and Q(0) == -2 and Q(1) == 0
assert R(64) == 0 and A(0) == 0 and A(1) == 0 and Q(0) == 0 and Q(1) == 0 and A(0) == 0
""")
