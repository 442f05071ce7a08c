"""What the orthogonalised update's launches read and write, worked out from the plan that each of them is given: no element outside its operand, no operand
outside the scratch that the call asks for.  No GPU: the library runs on the recorder, whose launches do nothing."""
import json
import os
import shutil
import subprocess
import sys
import textwrap

import pytest

from tests.test_dispatch_cpu import HERE, PRELUDE, ROOT

READER = """
import re
rec.recorder_plan.restype = ctypes.c_char_p


def plans(call):
    # (kernel, its integer template arguments, workgroups, plan, groups) of every launch
    found = []
    for i, name in enumerate(launches(call)):
        lines = [line.split() for line in rec.recorder_plan(i).decode().splitlines()]
        values = [{k: int(v) for k, v in zip(line[::2], line[1::2])} for line in lines]
        args = name.split("kernelI")[1] if "kernelI" in name else ""
        found.append((re.search(r"(muon|ns)_[a-z_]*kernel", name).group(), [int(v) for v in re.findall("L[ib]([0-9]+)E", args)], rec.recorder_grid(i, 0), values[0], values[1:]))
    return found


def eighths(v): return (v + 7) // 8 * 8


def wrong(call, nbytes):
    # what lies outside: (kernel, phase, what)
    bad = []
    def check(ok, *what):
        if not ok: bad.append([str(w) for w in what])
    for kernel, args, grid, p, groups in plans(call):
        check(p["bytes"] <= nbytes, kernel, "scratch", p["bytes"], nbytes)
        if p["tile"] == 3: continue
        ortho = [g for g in groups if g["ortho"]]
        # the operands lie one behind the other, inside the scratch
        planes = 2 if p["exact"] else 1
        at = 0
        for g in ortho:
            nx, ns = g["rp"] * g["cp"] * g["count"], g["mp"] ** 2 * g["count"]
            check(g["rp"] >= g["rows"] and g["cp"] >= g["cols"] and g["mp"] >= min(g["rows"], g["cols"]) and g["tall"] == (g["rows"] > g["cols"]), kernel, "sizes", g)
            check(g["xplane"] == nx and g["splane"] == ns, kernel, "planes", g)
            for key, n in (("x0", 2 * nx), ("x1", 2 * nx), ("s", planes * ns), ("b", planes * ns)):
                check(g[key] >= at, kernel, key, g)
                at = g[key] + n
        check(2 * at <= p["sums_at"], kernel, "halves")
        check(p["sums_at"] + 8 * sum(g["count"] * g["chunks"] for g in groups) <= p["diag_at"], kernel, "sums")
        check(p["diag_at"] + 4 * max(g["diag"] + 2 * g["count"] * g["mp"] for g in ortho) <= p["part_at"], kernel, "diagonals")
        if kernel == "muon_cast_kernel":
            check(all(g["casts"] * 4096 == g["rp"] * g["cp"] for g in ortho) and grid == sum(g["count"] * g["casts"] for g in ortho), kernel)
        if kernel != "ns_product_kernel": continue
        tm, tn, split, lo, low, phase, buffers, sets = args
        bm, bn, most = 64 * tm, 64 * tn, 0
        for g in ortho:
            inside = lambda what, edge, of: check(edge <= of, kernel, phase, what, edge, of, g)
            nt = 0
            while nt * (nt + 1) // 2 < g["grams"]: nt += 1
            check(nt * (nt + 1) // 2 == g["grams"], kernel, phase, "grams", g)
            # the longer side of X is what S is summed over
            along, across = (g["rp"], g["cp"]) if g["tall"] else (g["cp"], g["rp"])
            if phase == 0:
                inside("rows of X", nt * bm, across); inside("rows of S", nt * bm, g["mp"])
                check(along % 64 == 0 and along >= max(g["rows"], g["cols"]), kernel, phase, "contraction", g)
                check(nt * bm >= min(g["rows"], g["cols"]), kernel, phase, "S is whole", g)
                if g["splits"] > 1: inside("parts", p["part_at"] + 4 * (g["part"] + g["count"] * g["grams"] * g["splits"] * bm * bm), nbytes)
                units = g["count"] * g["grams"] * g["splits"]
            elif phase == 1:
                inside("rows of S", nt * bm, g["mp"]); inside("columns of S", (g["mp"] + 63) // 64 * 64, g["mp"])
                units = g["count"] * g["grams"]
            else:
                nc = g["cp"] // bn
                check(g["applies"] % nc == 0, kernel, phase, "tiles", g)
                rows, cols = g["applies"] // nc * bm, nc * bn
                inside("rows of X", rows, g["rp"]); inside("columns of X", cols, g["cp"])
                check(rows >= g["rows"] and cols >= g["cols"], kernel, phase, "X is whole", g)
                inside("rows of B and its diagonal", cols if g["tall"] else rows, g["mp"])
                inside("contraction, in X", (g["mp"] + 63) // 64 * 64, across); inside("contraction, in B", (g["mp"] + 63) // 64 * 64, g["mp"])
                # the last matrix's furthest element of B
                last = g["b"] + (planes - 1) * g["splane"] + (g["count"] - 1) * g["mp"] ** 2 + (cols if g["tall"] else rows) * g["mp"]
                inside("B in scratch", 2 * last, nbytes)
                units = g["count"] * g["applies"]
            most += eighths(units)
        check(grid == most, kernel, phase, "workgroups", grid, most)
    return bad


def orthogonalize(count, rows, cols, mode):
    n = bl.muon_orthogonalize_scratch_bytes(count, rows, cols, mode)
    return lambda: bl.muon_orthogonalize(P, P, count, rows, cols, mode, P, n, 0), n


def model(flags, *dims):
    c = bl.blstm_create(1, 1, *dims)
    n = bl.muon_scratch_bytes(c, flags)
    return lambda: bl.muon_step(c, P, P, P, P, 0.02, 0.1, 0.9, 0.1, flags, P, n, 0), n
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    out = str(tmp_path_factory.mktemp("plans") / "libplans.so")
    subprocess.run([gxx, "-O1", "-w", "-shared", "-fPIC", "-std=c++17", "-I", os.path.join(HERE, "wave_on_cpu"), "-I", os.path.join(ROOT, "paper_1904_04956_amd", "csrc"), "-o", out,
                    os.path.join(HERE, "muon_plans.cpp")], check=True)

    def run(code):
        text = PRELUDE.format(root=ROOT, recorder=out) + READER + textwrap.dedent(code) + "\nprint(json.dumps(out))\n"
        r = subprocess.run([sys.executable, "-c", text], capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr
        return json.loads(r.stdout.splitlines()[-1])
    return run


# sides on both sides of every multiple of 64, 128 and 256 that a tile can end at, and what lies between
SIDES = sorted({s for m in (128, 256, 384, 512, 640, 768, 1024, 1152, 1280, 2048, 2176, 4096) for s in (m - 1, m, m + 1)} | {65, 100, 300, 602, 1204, 1400, 2600, 3900, 4200})


@pytest.mark.parametrize("count", [1, 2, 7, 11, 32])
def test_matrices_lie_inside(plans, count):
    got = plans(f"""
        out = {{}}
        sides = {SIDES!r}
        pairs = {{(r, c) for r in sides for c in (r - 1, r, r + 1, r + 63, r + 100, r + 127, 2 * r, 65, 260, 1024) if 1 <= c <= 4300 and r * c * {count} < 1 << 27}}
        for r, c in sorted(pairs | {{(c, r) for r, c in pairs}}):
            for mode in (0, 1):
                bad = wrong(*orthogonalize({count}, r, c, mode))
                if bad: out[str(({count}, r, c, mode))] = bad[:2]
    """)
    assert got == {}


@pytest.mark.parametrize("sizes", [(1, 3900, 3900, 1), (3, 2600, 2600, 1), (24, 769, 769, 1), (4, 2100, 2100, 1), (8, 1600, 1600, 1), (16, 1100, 1100, 1), (8, 1300, 1400, 1), (300, 600, 640, 1)], ids=str)
def test_near_squares_on_tall_tiles_lie_inside(plans, sizes):
    tile, bad = plans(f"""
        call, n = orthogonalize(*{sizes})
        out = [plans(call)[0][3]["tile"], wrong(call, n)]
    """)
    assert tile == 2 and bad == []


@pytest.mark.parametrize("flags", [0, 2, 4, 7])
def test_models_lie_inside(plans, flags):
    got = plans(f"""
        out = {{}}
        for dims in ((260, 512, 4, 256, 32000), (260, 512, 6, 256, 32000), (260, 1024, 6, 256, 32000), (260, 301, 2, 67, 3001), (600, 700, 3, 300, 5000), (40, 32, 1, 0, 100), (40, 32, 5, 100, 100),
                     (64, 128, 2, 256, 3000), (1000, 130, 6, 512, 900), (300, 65, 1, 130, 30000), (260, 900, 1, 0, 3000), (2000, 257, 4, 500, 600), (515, 320, 6, 640, 32000)):
            for mode in (0, 1):
                bad = wrong(*model({flags}, *dims, mode))
                if bad: out[str((dims, mode))] = bad[:2]
    """)
    assert got == {}


@pytest.mark.parametrize("rows,cols", [(2 ** 31 - 1, 1), (1, 2 ** 31 - 1), (1, 2147483600), (2147483500, 1), (2 ** 30 + 1, 1), (1, 2 ** 30 + 1), (2 ** 31 - 1, 2 ** 8), (1, 2 ** 24)])
@pytest.mark.parametrize("mode", [0, 1])
def test_sides_that_no_padding_fits_are_refused(rows, cols, mode):
    from paper_1904_04956_amd import binding as bl
    for call in (lambda: bl.muon_orthogonalize_scratch_bytes(1, rows, cols, mode), lambda: bl.muon_orthogonalize(4096, 1 << 40, 1, rows, cols, mode, 4096, 1 << 62, 0),
                 lambda: bl.muon_matrices_step(4096, None, 4096, None, 1, rows, cols, mode, 0.1, 0.0, 0.0, 0, 4096, 1 << 62, 0)):
        with pytest.raises(bl.BlstmError) as e:
            call()
        assert e.value.code == -2
