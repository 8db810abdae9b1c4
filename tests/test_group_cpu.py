"""Refusals of the grouped operators, on the CPU: the C entry points' status
codes (nothing is enqueued) and the binding's own checks.  The plain 64-bit
forms that the GPU tests compare with are held against one another here."""
import itertools
import os
import re
import shutil
import subprocess

import pytest
import torch

import group_util as ref
from paper_2406_05955_amd import binding as ts

OK, NULL, SHAPE, DTYPE, ALIGN, WS, HIP, UNSUP = range(8)
A = 0x10000  # a 16-byte aligned fake device address; never dereferenced
lib = ts.lib


def mm(x=A, w=A, x2=None, w2=None, dt=1, kn=0, src=None, off=A, rows=8, S=8, G=2, n=16, k=16, out=A, odt=1):
    return lib.ts_grouped_mm(x, w, x2, w2, dt, kn, src, off, rows, S, G, n, k, out, odt, None)


def drelu(x=A, wg=A, wu=A, dt=1, src=None, off=A, rows=8, S=8, G=2, n=16, k=16, c=A, gate=None, up=None, odt=1):
    return lib.ts_grouped_drelu(x, wg, wu, dt, src, off, rows, S, G, n, k, c, gate, up, odt, None)


def dw(x=A, w=A, dt=1, src=None, off=A, rows=8, S=8, G=2, n=16, k=16, out=A, odt=1):
    return lib.ts_grouped_mm_dw(w, x, dt, src, off, rows, S, G, n, k, out, odt, None)


def fp8(x=A, xs=A, w=A, ws=A, src=None, off=A, rows=8, S=8, G=2, n=16, k=16, out=A, odt=1):
    return lib.ts_fp8_mm(x, xs, w, ws, src, off, rows, S, G, n, k, out, odt, None)


def fp8_drelu(x=A, wu=A, us=A, src=None, off=A, rows=8, S=8, G=2, n=16, k=16, out=A, odt=1):
    return lib.ts_fp8_drelu(x, A, A, A, wu, us, src, off, rows, S, G, n, k, out, odt, None)


@pytest.mark.parametrize("call", [mm, drelu, dw, fp8, fp8_drelu])
def test_products_refuse_sizes_and_pointers(call):
    for bad in (dict(rows=-1), dict(rows=(1 << 23) + 1, S=1 << 23), dict(G=0), dict(G=65), dict(n=0), dict(k=0),
                dict(n=12), dict(k=20), dict(n=1 << 18), dict(S=0), dict(S=7), dict(S=(1 << 23) + 1),
                dict(n=131072, k=131072)):
        assert call(**bad) == SHAPE, bad
    assert call(odt=3) == DTYPE
    assert call(off=None) == NULL
    assert call(off=A + 2) == ALIGN and call(src=A + 1, S=3) == ALIGN
    assert call(x=A + 8) == ALIGN and call(x=None) == NULL


def test_products_refuse_the_rest():
    assert mm(dt=2) == DTYPE and dw(dt=2) == DTYPE and drelu(dt=2) == DTYPE
    assert mm(w=None) == NULL and mm(out=None) == NULL and dw(out=None) == NULL and dw(w=None) == NULL
    assert mm(x2=A) == NULL and mm(w2=A) == NULL and mm(x2=A, w2=A + 4) == ALIGN and mm(out=A + 8) == ALIGN
    assert mm(dt=0, n=12, k=20, out=None) == NULL and mm(dt=0, n=14) == SHAPE
    assert drelu(gate=A) == NULL and drelu(up=A) == NULL and drelu(wu=None) == NULL and drelu(c=None) == NULL
    assert drelu(gate=A + 4, up=A) == ALIGN and drelu(wu=A + 2) == ALIGN
    assert fp8(xs=None) == NULL and fp8(ws=None) == NULL and fp8(xs=A + 2) == ALIGN and fp8(n=24) == SHAPE
    assert fp8_drelu(wu=None) == NULL and fp8_drelu(us=None) == NULL and fp8_drelu(wu=A + 8) == ALIGN


def test_no_rows_is_nothing_to_do():
    assert mm(rows=0, S=0, x=None, w=None, out=None) == OK
    assert drelu(rows=0, S=0, x=None, c=None) == OK
    assert fp8(rows=0, S=0, x=None, xs=None) == OK
    assert dw(rows=0, S=0, x=None, w=None, out=None) == NULL  # its zeros are written all the same
    assert lib.ts_drelu_grad(None, None, None, 1, 0, 16, None, None, None) == OK
    assert lib.ts_fp8_quant(None, 1, 0, 16, None, None, None) == OK
    assert lib.ts_moe_combine(None, 1, None, None, 0, 2, 16, 0, None, 1, None) == OK
    assert lib.ts_moe_route(None, 0, 8, 2, None, None, None, None, None, None, 0, None) == OK
    assert lib.ts_moe_route_grad(None, None, None, 0, 8, 2, None, None) == OK


def test_drelu_grad_and_quantisers():
    f = lib.ts_drelu_grad
    assert f(A, A, A, 5, 4, 16, A, A, None) == DTYPE
    assert f(A, A, A, 1, -1, 16, A, A, None) == SHAPE and f(A, A, A, 1, 4, 12, A, A, None) == SHAPE
    assert f(A, None, A, 1, 4, 16, A, A, None) == NULL and f(A, A, A, 1, 4, 16, A, None, None) == NULL
    assert f(A, A, A + 2, 1, 4, 16, A, A, None) == ALIGN
    q = lib.ts_fp8_quant
    assert q(A, 4, 4, 16, A, A, None) == DTYPE and q(A, 1, 4, 24, A, A, None) == SHAPE
    assert q(A, 1, -4, 16, A, A, None) == SHAPE and q(A, 1, 4, 16, None, A, None) == NULL
    assert q(A + 8, 1, 4, 16, A, A, None) == ALIGN and q(A, 1, 4, 16, A, A + 2, None) == ALIGN
    w = lib.ts_fp8_quant_weights
    assert w(A, 9, 0, 1, 16, 16, A, A, None) == DTYPE and w(A, 1, 0, 0, 16, 16, A, A, None) == SHAPE
    assert w(A, 1, 0, 1, 16, 8, A, A, None) == SHAPE and w(A, 1, 0, 1, 16, 16, A, None, None) == NULL


def test_routing():
    def route(l=A, T=8, E=8, K=2, idx=A, w=A, off=A, tok=A, pair=A, ws=A, n=1 << 20):
        return lib.ts_moe_route(l, T, E, K, idx, w, off, tok, pair, ws, n, None)
    for bad in (dict(T=-1), dict(E=0), dict(E=65), dict(K=0), dict(K=9, E=16), dict(K=3, E=2), dict(T=(1 << 22) + 1)):
        assert route(**bad) == SHAPE, bad
    assert route(l=None) == NULL and route(idx=None) == NULL and route(w=None) == NULL
    assert route(off=None) == NULL and route(tok=None) == NULL and route(pair=None) == NULL
    assert route(l=A + 2) == ALIGN and route(pair=A + 1) == ALIGN
    need = ts.moe_route_workspace_bytes(5000, 8, 2)
    assert need > 0 and ts.moe_route_workspace_bytes(-1, 8, 2) == 0
    assert route(T=5000, ws=None) == WS and route(T=5000, n=need - 1) == WS and route(T=5000, ws=A + 4, n=need) == ALIGN

    def group(idx=A, T=8, E=8, K=2, off=A, tok=A, pair=A, ws=A, n=1 << 20):
        return lib.ts_moe_group(idx, T, E, K, off, tok, pair, ws, n, None)
    assert group(T=-1) == SHAPE and group(idx=None) == NULL and group(off=None) == NULL and group(tok=None) == NULL
    assert group(off=A + 2) == ALIGN and group(T=5000, ws=None) == WS
    g = lib.ts_moe_route_grad
    assert g(A, A, A, 4, 65, 2, A, None) == SHAPE and g(A, None, A, 4, 8, 2, A, None) == NULL
    assert g(A, A, A + 2, 4, 8, 2, A, None) == ALIGN


def test_combine():
    def f(y=A, yd=1, pair=A, w=A, T=4, K=2, H=16, R=8, out=A, od=1):
        return lib.ts_moe_combine(y, yd, pair, w, T, K, H, R, out, od, None)
    for bad in (dict(T=-1), dict(K=0), dict(K=9), dict(H=12), dict(H=0), dict(R=-1), dict(H=1 << 18), dict(T=1 << 23)):
        assert f(**bad) == SHAPE, bad
    assert f(yd=2) == DTYPE and f(od=2) == DTYPE and f(y=None) == NULL and f(pair=None) == NULL and f(out=None) == NULL
    assert f(y=A + 8) == ALIGN and f(w=A + 2) == ALIGN

    def g(do=A, od=1, y=A, yd=1, pair=A, w=A, T=4, K=2, H=16, R=8, dy=A, dw_=A):
        return lib.ts_moe_combine_grad(do, od, y, yd, pair, w, T, K, H, R, dy, dw_, None)
    assert g(H=12) == SHAPE and g(od=7) == DTYPE and g(w=None) == NULL and g(dy=None) == NULL and g(dw_=None) == NULL
    assert g(do=A + 4) == ALIGN and g(dw_=A + 2) == ALIGN


def z(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype)


def test_binding_checks():
    i32, f32, e4 = torch.int32, torch.float32, torch.float8_e4m3fn
    x, w, off = z(8, 16), z(2, 24, 16), z(3, dtype=i32)
    for call, err in (
            (lambda: ts.grouped_mm(z(8, 16, dtype=torch.float16), w, off), TypeError),
            (lambda: ts.grouped_mm(x, w.float(), off), TypeError),
            (lambda: ts.grouped_mm(x, z(2, 24, 32), off), ValueError),
            (lambda: ts.grouped_mm(x, w, off, w_kn=True), ValueError),
            (lambda: ts.grouped_mm(x, w), ValueError),
            (lambda: ts.grouped_mm(x, w, z(4, dtype=i32)), ValueError),
            (lambda: ts.grouped_mm(x, w, off.long()), TypeError),
            (lambda: ts.grouped_mm(x, w, off, row_src=z(8, dtype=torch.int64)), TypeError),
            (lambda: ts.grouped_mm(z(0, 16), w, off, row_src=z(8, dtype=i32)), ValueError),
            (lambda: ts.grouped_mm(x, w, off, x2=x), ValueError),
            (lambda: ts.grouped_mm(x, w, off, x2=z(7, 16), w2=w), ValueError),
            (lambda: ts.grouped_mm(x, w, off, out_dtype=torch.float16), TypeError),
            (lambda: ts.grouped_mm(x, w, off), ValueError),  # host tensors
            (lambda: ts.grouped_drelu(x, w, z(2, 16, 16), off), ValueError),
            (lambda: ts.grouped_mm_dw(z(7, 24), x, off), ValueError),
            (lambda: ts.grouped_mm_dw(z(8, 24, dtype=f32), x, off), TypeError),
            (lambda: ts.drelu_grad(x, x, z(8, 24)), ValueError),
            (lambda: ts.fp8_quant(z(8, 16, dtype=torch.float16)), TypeError),
            (lambda: ts.fp8_mm(z(8, 16, dtype=e4), z(8, 2, dtype=f32), z(2, 24, 16, dtype=e4), z(2, 1, 1, dtype=f32), off),
             ValueError),
            (lambda: ts.fp8_mm(x, z(8, 1, dtype=f32), w, z(2, 1, 1, dtype=f32), off), TypeError),
            (lambda: ts.moe_route(z(8, 4, dtype=f32), 5), ValueError),
            (lambda: ts.moe_route(x, 2), TypeError),
            (lambda: ts.moe_group(z(8, 2, dtype=i32), 0), ValueError),
            (lambda: ts.moe_route_grad(z(8, 2, dtype=i32), z(8, 2, dtype=f32), z(8, 3, dtype=f32), 8), ValueError),
            (lambda: ts.moe_combine(x, z(4, 2, dtype=i32), z(4, 3, dtype=f32)), ValueError),
            (lambda: ts.moe_combine_grad(z(3, 16), x, z(4, 2, dtype=i32), z(4, 2, dtype=f32)), ValueError)):
        with pytest.raises(err):
            call()


def test_binding_refuses_extents_that_wrap():
    """The library's sizes are C ints: 2^32 + 8 rows would count as 8."""
    n, i32, f32 = 2 ** 32 + 8, torch.int32, torch.float32

    def wide(cols, dtype=torch.bfloat16):
        return torch.zeros(1, cols, dtype=dtype).expand(n, cols)  # (no memory)

    w, off = z(2, 24, 16), z(3, dtype=i32)
    for call in (lambda: ts.grouped_mm(wide(16), w, off), lambda: ts.grouped_drelu(wide(16), w, w, off),
                 lambda: ts.grouped_mm(z(8, 16), w, off, row_src=z(1, dtype=i32).expand(n)),
                 lambda: ts.grouped_mm_dw(wide(24), z(8, 16), off), lambda: ts.drelu_grad(wide(16), wide(16), wide(16)),
                 lambda: ts.fp8_quant(wide(16)), lambda: ts.fp8_quant_weights(z(1, 1, 16).expand(2, n, 16)),
                 lambda: ts.moe_route(wide(8, f32), 2), lambda: ts.moe_group(wide(2, i32), 8),
                 lambda: ts.moe_group(z(8, 2, dtype=i32), n), lambda: ts.moe_combine(z(8, 16), wide(2, i32)),
                 lambda: ts.moe_combine(wide(16), z(8, 2, dtype=i32)),
                 lambda: ts.moe_route_grad(z(8, 2, dtype=i32), z(8, 2, dtype=f32), z(8, 2, dtype=f32), n)):
        with pytest.raises(ValueError, match=r"2\^31"):
            call()


def test_weight_gradient_without_rows_still_checks_its_offsets():
    assert dw(rows=0, x=None, w=None, off=A + 2) == ALIGN


# --- the plain forms ---------------------------------------------------------------

def test_plain_products_against_loops():
    g = torch.Generator().manual_seed(1)
    x, w = torch.randn(9, 5, generator=g), torch.randn(3, 4, 5, generator=g)
    off, src = torch.tensor([1, 4, 4, 8]), torch.tensor([8, 0, 3, 3, 1, 2, 7, 5, 6])
    y, mag = ref.mm(x, w, off, src)
    d, _ = ref.dw(y.nan_to_num(0).float(), x, off, src)
    assert torch.isnan(y[[0, 8]]).all() and (d[1] == 0).all()
    for e, r in ((0, 1), (0, 2), (0, 3), (2, 4), (2, 7)):
        for j in range(4):
            terms = [float(x[src[r], i]) * float(w[e, j, i]) for i in range(5)]
            assert abs(sum(terms) - y[r, j]) < 1e-12 and abs(sum(map(abs, terms)) - mag[r, j]) < 1e-12
    assert torch.allclose(d[2], sum(y[r].float().double()[:, None] * x[src[r]].double() for r in range(4, 8)))


def test_plain_routing_against_all_choices():
    """Top-k as the best of all ordered choices; rows by counting."""
    l = torch.tensor([[1.0, 3.0, 3.0, 2.0], [float("nan"), -float("inf"), 0.0, 0.0]])
    idx, w, off, tok, pair = ref.route(l, 2)
    for t in range(2):
        v = [-float("inf") if a != a else a for a in l[t].tolist()]
        best = max(itertools.permutations(range(4), 2), key=lambda c: [(v[i], -i) for i in c])
        assert idx[t].tolist() == list(best)
    assert idx.tolist() == [[1, 2], [2, 3]] and torch.allclose(w, torch.full((2, 2), 0.5, dtype=ref.D))
    assert off.tolist() == [0, 0, 1, 3, 4] and tok.tolist() == [0, 0, 1, 1] and pair.tolist() == [[0, 1], [2, 3]]


def test_plain_quantiser():
    """Every e4m3 value times a power of two keeps its code; scales as defined."""
    v = torch.arange(256, dtype=torch.uint8).view(ref.E4M3).float()
    v = v[torch.isfinite(v)]
    x = torch.zeros(1, 384)
    x[0, :254] = v[:254]
    x[0, 254] = x[0, 0:1].new_tensor(448.0)
    x[0, 0] = 448.0
    q, s = ref.quant_rows(x)
    assert torch.equal(ref.row_values(q, s).float(), x)
    assert s.tolist()[0][:2] == [1.0, 1.0]


@pytest.mark.parametrize("T,E,K,H,I", ref.FP8_LAYERS)
def test_plain_fp8_layer_tells_mistakes(T, E, K, H, I):
    """The bounds of the 8-bit layer take the layer itself, with Combined, the
    down product and the output rounded as they are passed on, and no layer
    with a scale, an expert, a column or a weight in the wrong place."""
    x, wr, wg, wu, wd = ref.fp8_layer_inputs(T, E, H, I, torch.Generator().manual_seed(T))
    logits = x.float() @ wr.float().t()
    gate, up, down = (ref.quant_tiles(m) for m in (wg, wu, wd.transpose(1, 2)))
    idx, w, off, tok, pair = ref.route(logits, K)
    xv = ref.row_values(*ref.quant_rows(x))
    g, u = (ref.mm(xv, ref.tile_values(*q), off, tok)[0] for q in (gate, up))
    c = ref.drelu(g, u).to(ref.BF16)
    y = ref.mm(ref.row_values(*ref.quant_rows(c)), ref.tile_values(*down), off)[0].to(ref.BF16)
    out = (w[:, :, None] * y.double()[pair.long()]).sum(1).to(ref.BF16)

    def holds(gate=gate, up=up, down=down, logits=logits, c_in=c, x=x):
        comb, comb_bound, want, bound = ref.fp8_layer(x, gate, up, down, logits, K, c_in)
        return bool(((c.double() - comb).abs() <= comb_bound).all() and ((out.double() - want).abs() <= bound).all())

    def scales(q, s):
        return q[0], s.contiguous()

    assert holds()
    cut = c.clone()
    cut[:, -16:] = 0
    for name, wrong in {
            "up: the first contraction block's scales": dict(up=scales(up, up[1][:, :, :1].expand_as(up[1]))),
            "gate: the first column block's scales": dict(gate=scales(gate, gate[1][:, :1].expand_as(gate[1]))),
            "down: the first column block's scales": dict(down=scales(down, down[1][:, :1].expand_as(down[1]))),
            "down: the first contraction block's scales": dict(down=scales(down, down[1][:, :, :1].expand_as(down[1]))),
            "up: another expert's scales": dict(up=scales(up, up[1].roll(1, 0))),
            "down: another expert's scales": dict(down=scales(down, down[1].roll(1, 0))),
            "the columns of Combined in another order": dict(c_in=c.flip(1)),
            "the last 16 columns of Combined left out": dict(c_in=cut),
            "x's neighbouring token": dict(x=x.roll(1, 0) if T > 1 else -x),
            "weights of 1 / K": dict(logits=logits.scatter(1, idx.long(), 9.0)),
    }.items():
        assert not holds(**wrong), name


# --- the host side's choices ---------------------------------------------------------

def build_check(tmp_path, *flags):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    csrc = os.path.join(root, "paper_2406_05955_amd", "csrc")
    exe = tmp_path / "group_check"
    subprocess.run(["g++", "-std=c++17", "-Wall", *flags, "-I", os.path.join(root, "include"), "-I", csrc,
                    os.path.join(root, "tests", "native", "group_check.cpp"), os.path.join(csrc, "ts_group.cpp"),
                    os.path.join(csrc, "ts_plan.cpp"), "-o", str(exe)], check=True)
    return exe


def test_host_side_under_sanitizers(tmp_path):
    exe = build_check(tmp_path, "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all")
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


def test_the_gpu_tests_reach_every_tile(tmp_path):
    """The shapes that the GPU tests take run every tile that the rule can
    choose: seven forward, six with dReLU (fp32: three of those)."""
    exe = build_check(tmp_path, "-O2")
    for kind, name in enumerate(("bf16", "f32", "fp8")):
        for drelu in (0, 1):
            lines = "\n".join(f"{kind} {drelu} {G} {rows} {n} {ref.TILE_K[name]}" for rows, G, n in ref.TILE_SHAPES)
            r = subprocess.run([str(exe), "-"], input=lines, capture_output=True, text=True, check=True)
            want = ({1, 2, 3} if name == "f32" else set(range(6))) | (set() if drelu else {6})
            assert set(map(int, r.stdout.split())) == want, (name, drelu)


def test_the_gpu_tests_of_many_scale_blocks_take_the_large_tile(tmp_path):
    exe = build_check(tmp_path, "-O2")
    rows, G, n = ref.EIGHTS
    lines = "\n".join(f"2 {drelu} {G} {rows} {n} {k}" for drelu in (0, 1) for k in ref.EIGHTS_K)
    r = subprocess.run([str(exe), "-"], input=lines, capture_output=True, text=True, check=True)
    assert set(map(int, r.stdout.split())) == {0}, r.stdout


def test_the_tile_table_fits_lds(tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = tmp_path / "tile_units_check"
    subprocess.run(["g++", "-std=c++17", "-Wall", "-I", os.path.join(root, "include"),
                    "-I", os.path.join(root, "paper_2406_05955_amd", "csrc"),
                    os.path.join(root, "tests", "native", "tile_units_check.cpp"), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout


def test_loads_written_out_read_scalar_copies():
    """A vector load written in assembler is invisible to the compiler's waits:
    it may read scalar registers only that its own text wrote with a scalar
    instruction (a vector instruction's take five issue slots until then), and
    m0 only one instruction after its write."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    csrc = os.path.join(root, "paper_2406_05955_amd", "csrc")
    found = 0
    for name in sorted(os.listdir(csrc)):
        if not name.endswith((".h", ".hip")):
            continue
        with open(os.path.join(csrc, name)) as f:
            text = f.read()
        for m in re.finditer(r'asm volatile\(\s*"([^"]*global_load_lds[^"]*)"', text):
            ops = m.group(1).split("\\n\\t")
            assert ops[0].startswith("s_mov_b32 m0") and len(ops) == 3, (name, ops)
            base = ops[-1].split()[-1]
            assert base == "off" or ops[1].startswith(f"s_mov_b64 {base},"), (name, ops)
            found += 1
    assert found >= 4


M0_KERNEL = """
#include "ts_gmm.h"
// the compiler's own loads into LDS, one before and one behind each written-out form
__global__ void probe(const char *p, float *o, uint32_t n) {
    __shared__ float s[4096];
    typedef __attribute__((address_space(3))) void lds;
    typedef const __attribute__((address_space(1))) void global;
    const auto own = [&] { __builtin_amdgcn_global_load_lds((global *)(p + threadIdx.x * 16), (lds *)s, 16, 0, 0); };
    for (uint32_t i = 0; i < n; ++i) {
        own();
        ts::ld_lds16(p + threadIdx.x * 16, 1024u);
        own();
        ts::ld_lds16(p, threadIdx.x * 16, 2048u);
        own();
        ts::ld_lds4(p, threadIdx.x * 4, 5120u);
        own();
        ts::ld_lds4(p, (size_t)threadIdx.x * 4, 6144u);
        own();
        __syncthreads();
    }
    o[threadIdx.x] = s[threadIdx.x] + s[threadIdx.x + 1024];
}
"""


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs the device compiler")
def test_loads_written_out_declare_m0(tmp_path):
    """A written-out load sets m0: the compiler is told (as a clobber it takes no
    note of a reserved register, and says so), and sets its own value again
    before its next use."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "m0.hip"
    src.write_text(M0_KERNEL)
    r = subprocess.run(["hipcc", "-O3", "-std=c++17", "--offload-arch=gfx950", "--offload-device-only", "-S", "-x", "hip",
                        "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                        "-I", os.path.join(root, "include"), "-I", os.path.join(root, "paper_2406_05955_amd", "csrc"),
                        str(src), "-o", str(tmp_path / "m0.s")], capture_output=True, text=True, check=True, timeout=300)
    assert "reserved register" not in r.stderr, r.stderr
    stale, inside, own, written = True, False, 0, 0
    for line in (tmp_path / "m0.s").read_text().splitlines():
        inside = (inside or "#ASMSTART" in line) and "#ASMEND" not in line
        if line.startswith(".LBB"):
            stale = True  # (a loop's start: what its end left)
        if "s_mov_b32 m0" in line:
            stale = inside
        if "global_load_lds" in line:
            assert inside or not stale, line
            written, own = written + inside, own + (not inside)
    assert written == 4 and own == 5
