"""The projection with adapters in tiles of 256 columns (gen_gemm_rows.py, gemm_adapted.hip): the generated part that adds the adapters followed on the CPU
with numbers, what it leaves alone, its wait states, and products on the GPU."""
import importlib.util
import os
import re
import subprocess
import sys

import numpy as np
import pytest

from tests import test_gemm_rows as G
from tests import test_wait_states as WS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
rows = G.rows
U32 = 0xffffffff
LOW_AT, UP_AT, INDEX_AT = 1 << 40, 3 << 41, 5 << 39


class _Wave:
    """One wave between two tiles: scalars as integers, vector registers as 64 integers, fragments as 64 x 8 numbers, sums as numbers"""
    def __init__(self, mt, wave, text, M, N, rank, adapters, tile, index, low, up, seed):
        self.mt, self.text, self.M, self.N, self.rank, self.adapters = mt, text, M, N, rank, adapters
        self.index, self.low, self.up = index, low, up
        self.label = {ln[:-1]: k for k, ln in enumerate(text) if ln.endswith(":")}
        self.arg = {"M": M, "N": N, "wave": wave, "rank2": 2 * rank, "adapters": adapters, "index": INDEX_AT}
        for name, at in (("low", LOW_AT), ("up", UP_AT)):
            self.arg[name + "_lo"], self.arg[name + "_hi"] = at & U32, at >> 32
        self.s = {rows.S_T: tile[0], rows.S_T + 1: tile[1]}
        self.v, self.f, self.wrote = {}, {}, set()
        rng = np.random.default_rng(seed)
        # sums[ti][tj]: W's row 4 (lane / 16) + r, X's row lane % 16
        self.a = {r: rng.integers(-50, 50, 64).astype(float) for r in range(32 * mt)}
        self.loads = 0

    def val(self, x):
        if x.startswith("%["):
            return self.arg[x[2:-1]]
        if x == "vcc":
            return self.s["vcc"]
        if re.fullmatch(r"v\d+", x):
            return self.v[int(x[1:])]
        if x.startswith("s["):
            lo = self.s[int(x[2:].split(":")[0])]
            return lo if isinstance(lo, np.ndarray) else lo | self.s[int(x[2:].split(":")[0]) + 1] << 32
        if re.fullmatch(r"s\d+", x):
            return self.s[int(x[1:])]
        return int(x, 0) & U32

    def put(self, d, x):
        n = int(d[1:])
        self.wrote.add(("v", n))
        self.v[n] = np.broadcast_to(np.asarray(x), 64).copy()

    def run(self):
        signed = lambda x: np.where(np.asarray(x) & 0x80000000, np.asarray(x, dtype=np.int64) - (1 << 32), x)      # noqa: E731
        k, scc, steps, flying = 0, 0, 0, set()
        self.flying = flying                                         # fragments asked for and not waited for
        lane = np.arange(64)
        while k < len(self.text):
            ln = self.text[k]
            k, steps = k + 1, steps + 1
            assert steps < 100000
            if ln.endswith(":"):
                continue
            op, _, rest = ln.partition(" ")
            a = [x.strip() for x in re.split(r",(?![^\[]*\])", rest)]
            if op in ("s_nop",):
                continue
            if op == "s_waitcnt":
                flying.clear()
            elif op == "s_branch" or (op == "s_cbranch_scc1" and scc):
                k = self.label[a[0]]
            elif op == "s_cbranch_scc1":
                pass
            elif op == "s_cmp_eq_u64":
                scc = int(self.val(a[0]).all() if a[1] == "-1" else not self.val(a[0]).any())
                assert a[1] in ("-1", "0")
            elif op.startswith("s_cmp_"):
                x, y = self.val(a[0]), self.val(a[1])
                scc = int({"eq": x == y, "lt": x < y, "ge": x >= y}[op.split("_")[2]])
            elif op.startswith("s_"):
                x, y = self.val(a[1]), self.val(a[2]) if len(a) > 2 else None
                if op in ("s_add_u32", "s_addc_u32"):
                    r = x + y + (scc if op == "s_addc_u32" else 0)
                    scc = r >> 32
                else:
                    r = {"s_mov_b32": lambda: x, "s_mul_i32": lambda: x * y, "s_mul_hi_u32": lambda: x * y >> 32, "s_sub_u32": lambda: x - y,
                         "s_lshl_b32": lambda: x << y, "s_lshr_b32": lambda: x >> y, "s_and_b32": lambda: x & y}[op]()
                    if op == "s_sub_u32":
                        scc = int(r < 0)
                n = int(a[0][1:])
                assert n >= 74, ln                                   # the stream's own scalars stay
                self.s[n] = r & U32
            elif op in ("v_mbcnt_lo_u32_b32", "v_mbcnt_hi_u32_b32"):
                self.put(a[0], lane if op.startswith("v_mbcnt_lo") else self.v[int(a[2][1:])])
            elif op == "v_bfrev_b32":
                assert a[1] == "-2"
                self.put(a[0], 0x7fffffff)
            elif op in ("v_cmp_ge_u32", "v_cmp_gt_u32", "v_cmp_lt_i32", "v_cmp_eq_u32"):
                x, y = np.asarray(self.val(a[1])), np.asarray(self.val(a[2]))
                if op.endswith("i32"):
                    x, y = signed(x), signed(y)
                r = np.broadcast_to({"ge": x >= y, "gt": x > y, "lt": x < y, "eq": x == y}[op.split("_")[2]], 64)
                self.s["vcc" if a[0] == "vcc" else int(a[0][2:].split(":")[0])] = r
            elif op == "v_cndmask_b32" or op == "v_cndmask_b32_e64":
                self.put(a[0], np.where(self.val(a[3]), self.val(a[2]), self.val(a[1])))
            elif op == "v_min_i32_dpp":
                assert a[0] == a[1] == a[2].split()[0] and "row_mask:0xf bank_mask:0xf" in ln
                x = signed(self.v[int(a[0][1:])])
                how = a[2].split()[1]
                if how.startswith("quad_perm"):
                    perm = [int(q) for q in re.search(r"\[(.*)\]", ln).group(1).split(",")]
                    of = (lane & ~3) + np.array(perm)[lane & 3]
                else:
                    of = (lane & ~7) + 7 - (lane & 7) if how == "row_half_mirror" else (lane & ~15) + 15 - (lane & 15)
                self.put(a[0], np.minimum(x, x[of]) & U32)
            elif op == "v_readfirstlane_b32":
                self.s[int(a[0][1:])] = int(self.v[int(a[1][1:])][0])
            elif op == "global_load_dword":
                at = self.val(a[2].split()[0]) + self.v[int(a[1][1:])] - INDEX_AT
                assert (at >= 0).all() and (at + 4 <= 4 * self.M).all() and (at % 4 == 0).all()
                self.put(a[0], self.index[at // 4].astype(np.int64) & U32)
            elif op == "global_load_dwordx4":
                d = int(a[0][2:].split(":")[0])
                assert 64 <= d < 128 and d % 4 == 0
                at = self.val(a[2]) + self.v[int(a[1][1:])].astype(object)
                from_, base = (self.up, UP_AT) if int(a[2][2:].split(":")[0]) == rows.S_UP else (self.low, LOW_AT)
                rel = np.array([int(x) - base for x in at])
                flat = from_.reshape(-1)
                assert (rel >= 0).all() and (rel % 16 == 0).all() and (rel + 16 <= 2 * flat.size).all(), ln
                self.f[d] = flat[rel[:, None] // 2 + np.arange(8)]
                self.loads += from_ is self.up
                flying.add(d)
            elif op.startswith("v_mfma"):
                d, fa, fb = (int(x[2:].split(":")[0]) for x in a[:3])
                assert fa not in flying and fb not in flying and 64 <= fa < 96 <= fb < 128
                A, Bm = np.zeros((16, 32)), np.zeros((32, 16))
                for q in range(64):
                    A[q & 15, (q >> 4) * 8:(q >> 4) * 8 + 8] = self.f[fa][q]
                    Bm[(q >> 4) * 8:(q >> 4) * 8 + 8, q & 15] = self.f[fb][q]
                with np.errstate(invalid="ignore"):
                    D = A @ Bm
                for r in range(4):
                    got = D[4 * (lane >> 4) + r, lane & 15]
                    if a[0].startswith("a["):
                        assert a[3] == a[0]
                        self.a[d + r] = self.a[d + r] + got
                    else:
                        assert a[3] == "0" and rows.ASUM <= d <= rows.ASUM + 12
                        self.v[d + r] = got
                        self.wrote.add(("v", d + r))
            elif op == "v_accvgpr_read_b32":
                self.put(a[0], self.a[int(a[1][1:])])
            elif op == "v_accvgpr_write_b32":
                self.a[int(a[0][1:])] = self.v[int(a[1][1:])].copy()
            elif op == "v_min_i32":
                self.put(a[0], np.minimum(signed(self.val(a[1])), signed(self.val(a[2]))) & U32)
            elif op == "v_add_f32":
                self.put(a[0], self.v[int(a[1][1:])] + self.v[int(a[2][1:])])
            else:
                x, y = np.asarray(self.val(a[1]), dtype=np.int64), np.asarray(self.val(a[2]), dtype=np.int64)
                if op == "v_mul_u32_u24":
                    assert (x < 1 << 24).all() and (y < 1 << 24).all()
                r = {"v_add_u32": lambda: x + y, "v_min_u32": lambda: np.minimum(x, y), "v_mul_u32_u24": lambda: x * y, "v_and_b32": lambda: x & y,
                     "v_lshrrev_b32": lambda: y >> x, "v_lshlrev_b32": lambda: y << x}[op]()
                assert (r < 1 << 32).all()
                self.put(a[0], r)


# rows, columns, rank, adapters, tile, which rows have which
FOLLOWED = [(300, 520, 32, 3, (1, 2), "runs"), (300, 520, 64, 3, (0, 1), "mixed"), (257, 8, 128, 2, (1, 0), "mixed"), (512, 256, 32, 1, (0, 0), "one"), (600, 264, 32, 5, (1, 1), "none"),
            (300, 776, 64, 4, (0, 3), "infinite")]


@pytest.mark.parametrize("wave", range(4))
@pytest.mark.parametrize("mt", [8, 6, 4])
@pytest.mark.parametrize("M,N,rank,adapters,tile,how", FOLLOWED)
def test_adapters_join_the_sums(mt, wave, M, N, rank, adapters, tile, how):
    """Whole numbers, whose sums are exact: each element of the tile gains its row's T times its adapter's row of its column, once; every load lies inside its
    operand and is waited for; registers that the stream of stages goes on with stay."""
    text = [ln.replace("_%=", "") for ln in rows.adapter_lines(mt)]
    rng = np.random.default_rng(mt + M)
    index = {"runs": np.arange(M) * adapters // M, "mixed": rng.integers(-1, adapters + 1, M), "one": np.zeros(M, int), "none": np.full(M, -1),
             "infinite": rng.integers(0, adapters, M)}[how]
    if how == "mixed":
        index[::5] = rng.choice([-2 ** 31, 2 ** 31 - 1, adapters], len(index[::5]))
        index[32:64] = 1
    low, up = rng.integers(-4, 5, (M, rank)).astype(float), rng.integers(-4, 5, (adapters, N, rank)).astype(float)
    if how == "infinite":
        up[1] = np.inf
        index[16:48] = 0                                             # (whole sub-tiles take the short way)
    w = _Wave(mt, wave, text, M, N, rank, adapters, tile, index, low, up, 3)
    before = {r: x.copy() for r, x in w.a.items()}
    w.run()
    lane = np.arange(64)
    for ti in range(8):
        for tj in range(mt):
            for r in range(4):
                m = 32 * mt * tile[0] + (wave & 1) * 16 * mt + 16 * tj + (lane & 15)
                n = 256 * tile[1] + (wave >> 1) * 128 + 32 * (ti // 2) + 8 * (lane >> 4) + 4 * (ti % 2) + r
                for q in np.flatnonzero((m < M) & (n < N)):
                    g = index[m[q]]
                    with np.errstate(invalid="ignore"):
                        add = low[m[q]] @ up[g, n[q]] if 0 <= g < adapters else 0.0
                    got = w.a[4 * (mt * ti + tj) + r][q]
                    want = before[4 * (mt * ti + tj) + r][q] + add
                    assert got == want or (np.isnan(got) and np.isnan(want)) or (g == 1 and how == "infinite" and not np.isfinite(got)), (ti, tj, r, q)
    assert all(64 <= n < 128 or rows.INDEX <= n <= rows.LAST_VGPR_ADAPTED for kind, n in w.wrote)
    if how == "one" and 32 * mt * tile[0] + (wave & 1) * 16 * mt < M:
        assert w.loads == 8 * rank // 32                             # an adapter that all rows have is loaded once


@pytest.mark.parametrize("mt", [8, 6, 4])
@pytest.mark.parametrize("rank", [32, 128])
@pytest.mark.parametrize("of", [set(), {0}, {70}, {0, 200}, {299}])
def test_no_load_is_left_on_its_way(mt, rank, of):
    """Whatever rows have an adapter, none included: a fragment that arrives behind the end would overwrite what the tile's results are in by then"""
    text = [ln.replace("_%=", "") for ln in rows.adapter_lines(mt)]
    index = np.array([1 if m in of else -1 for m in range(300)])
    for wave in range(4):
        for tile in range(-(-300 // (32 * mt))):
            w = _Wave(mt, wave, text, 300, 256, rank, 2, (tile, 0), index, np.zeros((300, rank)), np.zeros((2, 256, rank)), 3)
            w.run()
            assert not w.flying, (wave, tile)


@pytest.mark.parametrize("mt", [8, 6, 4])
def test_the_rest_is_the_plain_program(mt):
    text, plain, part = (list(x) for x in (rows.generate(mt, "adapted"), rows.generate(mt), rows.adapter_lines(mt)))
    at = text.index(part[0])
    assert text[at:at + len(part)] == part
    del text[at:at + len(part)]
    assert text == plain
    # ... behind the end of the last products, and where nothing but the next tile's first stage is held: X in set 0, W's first rows
    full = rows.generate(mt, "adapted")
    assert full[full.index(part[0]) - 1] == "s_nop 3" and "s_nop 15" in full[full.index(part[0]) - 6:full.index(part[0])]


@pytest.mark.parametrize("mt", [8, 6, 4])
def test_wait_states(mt):
    assert WS.too_close(rows.generate(mt, "adapted")) == []


def test_kernels_do_not_spill(tmp_path):
    spec = importlib.util.spec_from_file_location("_flags", os.path.join(ROOT, "paper_2511_20426_amd", "_build.py"))
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)
    subprocess.run([sys.executable, os.path.join(build.CSRC, "gen_gemm_rows.py"), str(tmp_path / "gemm_rows_gfx950.inc")], check=True, capture_output=True)
    out = tmp_path / "out.s"
    subprocess.run([build.hipcc(), "-x", "hip", "-S", "--offload-device-only", os.path.join(build.CSRC, "gemm_adapted.hip"), "-o", str(out), "-O3", "-std=c++17",
                    "--offload-arch=gfx950", "-I", os.path.join(ROOT, "include"), "-I", build.CSRC, "-I", str(tmp_path)] + build.DEVICE_FLAGS, check=True,
                   capture_output=True)
    text = out.read_text()
    names = re.findall(r"\.name:\s*(\S*_kernel\S*)", text)
    spilled = [int(n) for n in re.findall(r"\.[sv]gpr_spill_count:\s*(\d+)", text)]
    assert len(names) >= 20 and len(spilled) == 2 * len(names) and not any(spilled), list(zip(names, spilled[::2], spilled[1::2]))


# tiles of 256, 192 and 128 rows, several to a workgroup and a last round, rows and columns past the end; ranks of one, two and four steps
PRODUCTS = [(5000, 2560, 128, 3, 32, "runs"), (3000, 4104, 256, 5, 64, "mixed"), (8300, 2056, 128, 4, 128, "mixed"), (8300, 2056, 128, 2, 20, "runs"),
            (4681, 1536, 1152, 5, 32, "runs"), (4681, 1544, 1152, 3, 100, "mixed"), (4800, 1536, 1152, 1, 32, "runs"), (9000, 1544, 256, 7, 16, "none")]


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,g,r,how", PRODUCTS)
def test_products(m, n, k, g, r, how):
    import torch

    from paper_2511_20426_amd.runner import Adapters, linear, linear_adapted
    from tests import test_adapters as T
    x, w, down, up, scales, index, _ = T._case(m, n, k, g, r, how)
    adapters = Adapters.from_weights(down, up, scales)
    y = linear_adapted(x, w, adapters, index)
    ref, _, off = T._adapted(x, w, down, up, scales, index)
    T._close(y, ref, off)
    none = (index < 0) | (index >= g)
    assert torch.equal(y[none], linear(x, w)[none])
    up2 = up.clone()
    up2[0, 5] = float("inf")                                         # one adapter's infinity is its rows' alone
    again = linear_adapted(x, w, Adapters.from_weights(down, up2, scales), index)
    assert torch.equal(again[index != 0], y[index != 0])
