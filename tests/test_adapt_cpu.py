"""Adapters beside a projection: what the host refuses, workspace sizes, the
tiles that the GPU tests reach."""
import os
import subprocess

import pytest
import torch

import adapt_util as ref
from paper_2406_05955_amd import binding as ts

OK, NULL, SHAPE, DTYPE, ALIGN, WS, HIP, UNSUP = range(8)
A = 0x10000


def _mm(x=A, w=A, a=A, b=A, scale=None, dt=1, kn=0, off=A, ad=A, rows=10, S=3, N=4, rank=16, n=64, k=64, out=A, odt=1, ws=A,
        wsb=1 << 40):
    return ts.lib.ts_adapter_mm(x, w, a, b, scale, dt, kn, off, ad, rows, S, N, rank, n, k, out, odt, ws, wsb, None)


def _dr(x=A, w=A, wu=A, a=A, b=A, au=A, bu=A, scale=None, dt=1, off=A, ad=A, rows=10, S=3, N=4, rank=16, n=64, k=64, out=A,
        odt=1, ws=A, wsb=1 << 40):
    return ts.lib.ts_adapter_drelu(x, w, wu, a, b, au, bu, scale, dt, off, ad, rows, S, N, rank, n, k, out, odt, ws, wsb, None)


@pytest.mark.parametrize("call", [_mm, _dr])
def test_refusals(call):
    assert call(dt=2) == DTYPE and call(odt=-1) == DTYPE
    for bad in (dict(n=60), dict(k=60), dict(n=0), dict(rank=0), dict(rank=12), dict(rank=136), dict(dt=0, rank=6), dict(N=0),
                dict(S=-1), dict(rows=-1), dict(rows=(1 << 23) + 1), dict(S=(1 << 23) + 1), dict(N=(1 << 23) + 1),
                dict(n=1 << 16, k=1 << 15)):
        assert call(**bad) == SHAPE, bad
    for name in ("x", "w", "a", "b", "off", "ad", "out"):
        assert call(**{name: None}) == NULL, name
        assert call(**{name: A + 2}) == ALIGN, name
    assert call(scale=A + 2) == ALIGN
    assert call(ws=None) == WS and call(wsb=16) == WS and call(ws=A + 4) == ALIGN
    assert call(rows=0, x=None) == OK and call(S=0, out=None) == OK


def test_refusals_of_up():
    for name in ("wu", "au", "bu"):
        assert _dr(**{name: None}) == NULL and _dr(**{name: A + 8}) == ALIGN


def test_workspace():
    size = lambda *a: ts.lib.ts_adapter_workspace_bytes(*a)  # noqa: E731
    one = size(100, 16, 1, 0, 64, 64, 1, 1)
    assert one >= 100 * 16 * 2 + 400
    assert size(100, 16, 2, 0, 64, 64, 1, 1) >= one + 100 * 16 * 2 - 256
    assert size(100, 16, 1, 0, 64, 64, 1, 0) == size(100, 16, 2, 0, 64, 64, 1, 1)
    assert size(100, 16, 1, 0, 64, 64, 0, 0) >= 100 * 16 * 4 + 400
    for bad in ((100, 16, 3, 0, 64, 64, 1, 1), (100, 12, 1, 0, 64, 64, 1, 1), (-1, 16, 1, 0, 64, 64, 1, 1), (100, 16, 1, 0, 64, 64, 2, 1),
                (100, 132, 1, 0, 64, 64, 0, 0), (100, 16, 1, 0, 60, 64, 1, 1), (100, 16, 1, 0, 64, 0, 1, 1)):
        assert size(*bad) == 0
    assert _mm(wsb=size(10, 16, 1, 0, 64, 64, 1, 1) - 1) == WS and _mm(odt=0, wsb=size(10, 16, 1, 0, 64, 64, 1, 1)) == WS


def test_binding_refuses_tensors():
    x, w, a, b = torch.zeros(4, 64), torch.zeros(32, 64), torch.zeros(3, 8, 64), torch.zeros(3, 32, 8)
    off, ad = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="contiguous device"):
        ts.adapter_mm(x, w, a, b, off, ad)
    for args in ((x, w, a, b[:2], off, ad), (x, w, a, b.transpose(1, 2), off, ad), (x, w[:, :32], a, b, off, ad),
                 (x, w, a[:, :, :32], b, off, ad), (x, w, a, b, off[:2], ad), (x, w[None], a, b, off, ad)):
        with pytest.raises(ValueError):
            ts.adapter_mm(*args)
    for args in ((x.bfloat16(), w, a, b, off, ad), (x, w, a, b, off.long(), ad), (x, w, a, b, off, ad.long())):
        with pytest.raises(TypeError):
            ts.adapter_mm(*args)
    with pytest.raises(ValueError, match="scale"):
        ts.adapter_mm(x, w, a, b, off, ad, scale=torch.zeros(2))
    with pytest.raises(ValueError, match="b must be"):
        ts.adapter_mm(x, w.t().contiguous(), a, b, off, ad, w_kn=True)
    with pytest.raises(ValueError, match="a_up"):
        ts.adapter_drelu(x, w, w, a, b, a[:, :4], b, off, ad)
    with pytest.raises(ValueError, match="b_up"):
        ts.adapter_drelu(x, w, w, a, b, a, b[:, :16], off, ad)


def build_tile_check(tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    csrc, exe = os.path.join(root, "paper_2406_05955_amd", "csrc"), tmp_path / "adapt_tile_check"
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(root, "include"), "-I", csrc,
                    os.path.join(root, "tests", "native", "adapt_tile_check.cpp"), os.path.join(csrc, "ts_group.cpp"),
                    os.path.join(csrc, "ts_plan.cpp"), "-o", str(exe)], check=True)
    return str(exe)


def test_tile_choice(tmp_path):
    r = subprocess.run([build_tile_check(tmp_path)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


def test_the_gpu_tests_reach_every_tile(tmp_path):
    """Every tile that can be chosen, with the contraction in one workgroup and shared."""
    exe = build_tile_check(tmp_path)
    for kind in (0, 1):
        for drelu, w_kn in ((0, 0), (0, 1), (1, 0)):
            lines = "\n".join(f"{kind} {drelu} {w_kn} {rows} {n} {k}" for rows, n, k in ref.TILES)
            r = subprocess.run([exe, "-"], input=lines, capture_output=True, text=True, check=True)
            got = {(int(t), int(s) > 1) for t, s in (line.split() for line in r.stdout.splitlines())}
            tiles = {1, 2, 3, 6} if kind else {0, 2, 3, 4, 5, 6}
            want = {(t, s) for t in tiles - ({6} if drelu else set()) for s in (False, True)}
            assert want <= got, (kind, drelu, w_kn, want - got)


def test_the_gpu_tests_reach_every_split(tmp_path):
    """Every tile with every split that is chosen for it over a grid of sizes (as large as
    a test's matrices may be)."""
    exe = build_tile_check(tmp_path)
    grid = [(r, n, k) for r in (1, 8, 33, 64, 130, 200, 300, 500, 700, 1000, 1500, 2000, 3000, 6000)
            for n in (8, 144, 264, 528, 1040, 2064, 4112, 8208, 14336)
            for k in (136, 520, 1032, 2056, 4104, 8200, 14344, 28672, 57352)
            if r * n * k <= 6e10 and (r + n) * k <= 1.2e8 and r * n <= 2e7 and 4 * n * k < 1 << 32]
    for kind in (0, 1):
        for drelu, w_kn in ((0, 0), (0, 1), (1, 0)):
            got = []
            for sizes in (grid, ref.TILES + ref.SPLITS):
                lines = "\n".join(f"{kind} {drelu} {w_kn} {rows} {n} {k}" for rows, n, k in sizes)
                r = subprocess.run([exe, "-"], input=lines, capture_output=True, text=True, check=True)
                got.append(set(r.stdout.splitlines()))
            assert len(got[0]) > 10 and got[0] <= got[1], (kind, drelu, w_kn, got[0] - got[1])
