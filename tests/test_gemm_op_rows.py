"""The 8-bit linear map and the gated projections in tiles of 256 rows of W (gen_gemm_rows.py, gemm_op_rows.hpp): the generated programs
followed on the CPU over several tiles, their wait states, and that their kernels keep everything in registers."""
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
U32, X_AT, W_AT, Y_AT = G.U32, G.X_AT, G.W_AT, G.Y_AT
UP_AT, XS_AT, WS_AT, G_AT, U_AT = 7 << 36, 1 << 42, 1 << 43, 1 << 44, 1 << 45
KINDS = ("i8", "gated")


class _Value:
    """What a float register holds: the sums that went into it, and of each lane the scales of which row of X and of W."""
    def __init__(self, sums=(), xs=None, ws=None):
        self.sums, self.xs, self.ws = frozenset(sums), xs, ws

    def joined(self, o):
        assert (self.xs is None or o.xs is None) and (self.ws is None or o.ws is None)
        return _Value(self.sums | o.sums, self.xs if o.xs is None else o.xs, self.ws if o.ws is None else o.ws)


class _Wave:
    """One of the four waves of a workgroup, as gemm_op_rows_kernel sets it up."""
    def __init__(self, kind, mt, wave, text, lds, shape, tiles, pad, form, save):
        M, N, K = shape                                        # K: bytes of a row
        self.kind, self.mt, self.text, self.lds, self.shape, self.tiles, self.wave = kind, mt, text, lds, shape, tiles, wave
        self.gated = kind == "gated"
        self.cols = 128 if self.gated else 256
        self.label = {ln[:-1]: k for k, ln in enumerate(text) if ln.endswith(":")}
        self.ldx, self.ldw, self.ldy = K + 16 * pad, K + 32 * pad + (64 if self.gated and wave & 1 else 0), 2 * (N + 24 * pad)
        self.w_at = UP_AT if self.gated and wave & 1 else W_AT
        lane = np.arange(64, dtype=np.int64)
        l15, grp, wm, wn, rows_ = lane & 15, lane >> 4, wave & 1, wave >> 1, 32 * mt
        row, col = wm * 16 * mt + (l15 & 7), wn * self.cols // 2 + 32 * (l15 >> 3) + 8 * grp
        at_list = np.minimum(lane, len(tiles) - 1)
        ylane, tile_y, row8 = row * self.ldy + col * 2, rows_ * self.ldy, 8 * self.ldy
        g, u = (G_AT, U_AT) if save else (0, 0)
        self.arg = {"tile_x": self.ldx * rows_, "tile_w": self.ldw * self.cols, "ldw2": self.ldw, "ldx2": self.ldx, "M": M, "N": N,
                    "n_stages": K // 128, "tiles": len(tiles), "form": form, "wave": wave, "lds0": 0,
                    "list_m": np.array([t[0] for t in tiles])[at_list], "list_n": np.array([t[1] for t in tiles])[at_list],
                    "roww": (wave >> 1 if self.gated else wave) * 64 + (lane >> 3), "rowx": wave * 8 * mt + (lane >> 3),
                    "chunkw": ((lane & 7) ^ ((lane >> 4) & 1)) * 16, "chunkx": ((lane & 7) ^ (lane >> 4)) * 16,
                    "aw0": (wn * 128 + 8 * (l15 >> 2) + (l15 & 3)) * 128 + ((grp ^ (l15 >> 1)) << 4),
                    "ax0": (wm * 16 * mt + l15) * 128 + ((grp ^ (l15 >> 1)) << 4), "row": row, "col": col, "ylane_lo": ylane & U32, "ylane_hi": ylane >> 32,
                    "g": g, "blocks_n": -(-N // 32), "act0": _Value(), "act1": _Value()}
        for name, at in (("x", X_AT), ("w", self.w_at), ("y", Y_AT), ("tile_y", tile_y), ("row8", row8), ("xs", XS_AT), ("ws", WS_AT), ("g", g), ("u", u)):
            self.arg[name + "_lo"], self.arg[name + "_hi"] = at & U32, at >> 32
        self.s, self.v, self.a = {}, {}, {}
        self.scc, self.m0, self.exec = 0, None, np.ones(64, bool)
        self.queue, self.flying, self.held, self.barriers = [], [], {}, 0
        self.written, self.saved, self.written_at, self.forms = {}, {}, {}, {}
        self.tile = 0

    def val(self, x):
        x = x.strip()
        if x.startswith("%["):
            return self.arg[x[2:-1]]
        if x in ("vcc", "exec"):
            return self.s[x] if x == "vcc" else self.exec
        if re.fullmatch(r"v\d+", x):
            assert not any(int(x[1:]) in q[1] for q in self.queue if q[0] == "scale"), x      # a scale that has not arrived
            return self.v[int(x[1:])]
        if x.startswith("s["):
            a = int(x[2:].split(":")[0])
            return self.s[a] if isinstance(self.s[a], np.ndarray) else self.s[a] | self.s[a + 1] << 32
        if re.fullmatch(r"-?s\d+", x):
            return self.s[int(x.lstrip("-")[1:])]
        if "-" in x[1:]:
            p, q = x.split("-", 1)
            return self.label[p] - self.label[q]
        return _Value() if "." in x else int(x, 0) & U32

    def sum_at(self, acc, lane):
        """(row, column) of Y that an accumulator's sum belongs to in a lane, and whether it is the up projection's"""
        ti, tj, r = acc // 4 // self.mt, acc // 4 % self.mt, acc % 4
        tm, tn = self.tiles[self.a[acc][0]]
        up = self.gated and ti >= 4
        ti -= 4 * up
        n = self.cols * tn + (self.wave >> 1) * self.cols // 2 + 32 * (ti // 2) + 8 * (lane >> 4) + 4 * (ti % 2) + r
        return 32 * self.mt * tm + (self.wave & 1) * 16 * self.mt + 16 * tj + (lane & 15), n, up

    def run(self):
        signed = lambda u: u - (1 << 32) if u & 0x80000000 else u  # noqa: E731
        mt, (M, N, K), lds = self.mt, self.shape, self.lds
        per_tile, k, steps, lanes = 2 * (K // 128), 0, 0, np.arange(64)
        while k < len(self.text):
            ln = self.text[k]
            k, steps = k + 1, steps + 1
            assert steps < 400000
            if ln.endswith(":") or ln.startswith(";"):
                continue
            op, _, rest = ln.partition(" ")
            a = [x.strip() for x in re.split(r",(?![^\[]*\])", rest)]
            offset = re.search(r"offset:(\d+)", ln)
            imm = int(offset.group(1)) if offset else 0
            assert imm < (4096 if op.startswith("global") else 65536)
            if op == "s_barrier":
                assert not self.flying, ln
                self.barriers += 1
                yield
            elif op == "s_getpc_b64":
                self.s[int(a[0][2:].split(":")[0])], self.s[int(a[0][2:].split(":")[0]) + 1] = k, 0
            elif op == "s_setpc_b64":
                k = self.val(a[0])
                assert self.text[k].endswith(":")
            elif op == "s_branch" or (op == "s_cbranch_scc1" and self.scc):
                k = self.label[a[0]]
            elif op.startswith("s_cmp_"):
                x, y = self.val(a[0]), self.val(a[1])
                if op.endswith("i32"):
                    x, y = signed(x), signed(y)
                self.scc = int({"eq": x == y, "lg": x != y, "lt": x < y, "ge": x >= y}[op.split("_")[2]])
            elif op == "s_and_b64":
                self.exec = self.val(a[1]) & self.val(a[2])
            elif op == "s_mov_b64":
                assert a[0] == "exec"
                bits = (1 << 64) - 1 if a[1] == "-1" else self.val(a[1])
                assert bits in (0, (1 << 64) - 1)
                self.exec = np.full(64, bool(bits))
            elif op.startswith("s_") and op not in ("s_nop", "s_waitcnt", "s_cbranch_scc1"):
                x = self.val(a[1])
                y = self.val(a[2]) if len(a) > 2 else None
                if op in ("s_add_u32", "s_addc_u32"):
                    r = x + y + (self.scc if op == "s_addc_u32" else 0)
                    self.scc = r >> 32
                elif op in ("s_sub_u32", "s_subb_u32"):
                    r = x - y - (self.scc if op == "s_subb_u32" else 0)
                    self.scc = int(r < 0)
                else:
                    r = {"s_mov_b32": lambda: x, "s_mul_i32": lambda: x * y, "s_mul_hi_u32": lambda: (x * y) >> 32, "s_sub_i32": lambda: x - y,
                         "s_lshl_b32": lambda: x << y, "s_lshr_b32": lambda: x >> y, "s_min_u32": lambda: min(x, y), "s_and_b32": lambda: x & y,
                         "s_cselect_b32": lambda: x if self.scc else y}[op]()
                if a[0] == "m0":
                    self.m0 = r & U32
                else:
                    self.s[int(a[0][1:])] = r & U32
            elif op == "s_waitcnt":
                m = re.search(r"vmcnt\((\d+)\)", ln)
                if m:
                    assert int(m.group(1)) < 64
                    keep = int(m.group(1))
                    self.queue = self.queue[len(self.queue) - keep:] if keep else []
                m = re.search(r"lgkmcnt\((\d+)\)", ln)
                if m:
                    self.flying = self.flying[len(self.flying) - int(m.group(1)):] if int(m.group(1)) else []
            elif op == "v_readlane_b32":
                at = self.val(a[2])
                assert at < len(self.tiles)
                self.s[int(a[0][1:])] = int(self.val(a[1])[at])
            elif op == "v_cmp_gt_i32":
                r = np.broadcast_to(signed(self.val(a[1])) > self.val(a[2]), 64)
                self.s["vcc" if a[0] == "vcc" else int(a[0][2:].split(":")[0])] = r
            elif op == "global_load_lds_dwordx4":
                base, off = self.val(a[1]), self.val(a[0])
                assert (off >= 0).all() and (off < 1 << 31).all()
                addr, at = base + off, (self.m0 + 16 * np.arange(64)) // 16
                kind = 0 if base < W_AT else 2 if base >= UP_AT else 1
                rel, ld = addr - (X_AT, W_AT, UP_AT)[kind], self.ldw if kind else self.ldx
                row, byte = rel // ld, rel % ld
                assert (rel >= 0).all() and (row < (N if kind else M)).all() and (byte + 16 <= K).all() and (byte % 16 == 0).all()
                assert (lds.read_at[at] < self.barriers).all()
                lds.row[at], lds.chunk[at], lds.op[at], lds.visible[at] = row, byte // 16, kind, False
                self.queue.append(("lds", at))
            elif op.startswith("global_load_dword"):            # scales
                n, to = (4, int(a[0][2:].split(":")[0])) if op.endswith("x4") else (1, int(a[0][1:]))
                base, off = self.val(a[2].split()[0]), self.val(a[1])
                assert base in (XS_AT, WS_AT) and (off % 4 == 0).all() and self.exec.all()
                at = (off + imm) // 4
                assert (at >= 0).all() and (at + n <= (M if base == XS_AT else N)).all()
                for i in range(n):
                    self.v[to + i] = _Value(xs=at.copy()) if base == XS_AT else _Value(ws=at + i)
                self.queue.append(("scale", set(range(to, to + n))))
            elif op == "ds_bpermute_b32":
                addr, src = self.val(a[1]), self.val(a[2].split()[0])
                assert (addr % 4 == 0).all() and src.ws is None and self.exec.all()
                self.v[int(a[0][1:])] = _Value(xs=src.xs[(addr + imm) // 4 % 64])
                self.flying.append(int(a[0][1:]))
            elif op == "global_store_dwordx4" and a[1].startswith("a["):      # a projection, straight from the accumulators
                acc, addr = int(a[1][2:].split(":")[0]), self.val(a[2].split()[0]) + self.val(a[0]) + imm
                up = int(addr[0]) >= U_AT
                rel = addr - (U_AT if up else G_AT)
                assert (rel[self.exec] % 16 == 0).all() and (rel[self.exec] >= 0).all()
                for lane in np.flatnonzero(self.exec):
                    block, at = divmod(int(rel[lane]), 2048)
                    m, n = 16 * (block // -(-N // 32)) + at % 1024 // 16 % 16, 32 * (block % -(-N // 32)) + 8 * (at % 1024 // 256) + 4 * (at // 1024)
                    assert m < -(-M // 16) * 16 and (m, n, up) not in self.saved
                    for r in range(4):
                        assert self.a[acc + r][1] == per_tile and self.sum_at(acc + r, lane) == (m, n + r, up)
                    self.saved[m, n, up] = True
                self.queue.append(("store", ()))
            elif op == "global_store_dwordx4":
                data, row0 = int(a[1][2:].split(":")[0]), int(a[0][2:].split(":")[0])
                addr = self.v[row0] + (self.v[row0 + 1] << 32) + imm - Y_AT
                for lane in np.flatnonzero(self.exec):
                    m, n = int(addr[lane]) // self.ldy, int(addr[lane]) % self.ldy // 2
                    assert m < M and n + 8 <= N and n % 8 == 0 and (m, n) not in self.written
                    for e in range(8):
                        from_lane, pair = self.v[data + e // 2][lane]
                        v = pair[e % 2]
                        got = sorted(self.sum_at(acc, from_lane) for acc in v.sums)
                        assert all(self.a[acc][1] == per_tile for acc in v.sums)
                        assert got == [(m, n + e, False)] + [(m, n + e, True)] * self.gated
                        if not self.gated:
                            assert v.xs[from_lane] == m and v.ws[from_lane] == n + e
                    self.written[m, n] = True
                how = ln.split()[-1] if not ln.split()[-1].startswith("offset") else ""
                assert self.forms.setdefault(self.a[0][0], how) == how
                self.queue.append(("store", ()))
            elif op == "ds_read_b128":
                reg = int(a[0][2:].split(":")[0])
                at = (self.val(a[1].split()[0]) + imm) // 16
                assert lds.visible[at].all() and reg not in self.flying, (ln, steps)
                for g in range(4):
                    assert len(set((at[16 * g:16 * g + 16] % 16).tolist())) == 16
                lds.read_at[at] = np.maximum(lds.read_at[at], self.barriers)
                self.held[reg] = (lds.op[at].copy(), lds.row[at].copy(), lds.chunk[at].copy())
                self.flying.append(reg)
            elif op.startswith("v_mfma"):
                assert op == rows.MFMA[self.kind]
                acc, fa, fb = (int(x[2:].split(":")[0]) for x in a[:3])
                assert a[3] == a[0] and fa not in self.flying and fb not in self.flying
                tile, count = self.a[acc]
                chunk = (count // 2) * 8 + (count % 2) * 4 + (lanes >> 4)
                # A: row lane % 16 of the sub-tile is what lane group (lane % 16) / 4 has in accumulator lane % 4
                n, up = (np.array([self.sum_at(acc + (q & 3), (q & 12) << 2)[i] for q in lanes & 15]) for i in (1, 2))
                m = self.sum_at(acc, lanes)[0]
                for frag, kind, want in ((fa, 1 + up, np.minimum(n, N - 1)), (fb, 0, np.minimum(m, M - 1))):
                    o, row, ch = self.held[frag]
                    assert (o == kind).all() and (row == want).all() and (ch == chunk).all(), (ln, tile, count)
                for r in range(4):
                    self.a[acc + r] = (tile, count + 1)
            elif op == "v_accvgpr_write_b32":
                acc, done = int(a[0][1:]), self.a.get(int(a[0][1:]))
                assert a[1] == "0" and (done is None or done[1] == per_tile)
                self.a[acc] = (0 if done is None else done[0] + 1, 0)
            elif op == "v_accvgpr_read_b32":
                self.put(a[0], _Value({int(a[1][1:])}))
            elif op == "v_cvt_pk_bf16_f32":
                lo, hi = self.val(a[1]), self.val(a[2])
                self.held.pop(int(a[0][1:]) & ~3, None)
                self.v[int(a[0][1:])] = [(lane, (lo, hi)) for lane in range(64)]
                self.written_at[int(a[0][1:])] = steps
            elif op == "v_mov_b32_dpp":
                d, (x, *how) = int(a[0][1:]), a[1].split()
                mask = int(re.search(r"bank_mask:(0x\w+)", ln).group(1), 16)
                assert how[:2] == ["row_ror:8", "row_mask:0xf"] and steps - self.written_at[int(x[1:])] > 2
                old, new = self.v[int(x[1:])], list(self.v[d])
                for lane in range(64):
                    if mask >> (lane % 16 // 4) & 1:
                        new[lane] = old[lane & 48 | (lane + 8) & 15]
                self.v[d], self.written_at[d] = new, steps
            elif op == "v_mov_b32" and isinstance(self.v.get(int(a[1][1:]) if a[1][0] == "v" else -1), list):
                self.v[int(a[0][1:])], self.written_at[int(a[0][1:])] = self.v[int(a[1][1:])], steps
            elif op in ("v_cvt_f32_i32", "v_exp_f32", "v_rcp_f32", "v_med3_f32"):
                assert int(a[1][1:]) not in self.flying
                self.put(a[0], self.val(a[1]))
            elif op in ("v_mul_f32", "v_fma_f32", "v_add_f32"):
                at = [self.val(x) for x in a[1:]]
                assert not any(re.fullmatch(r"v\d+", x) and int(x[1:]) in self.flying for x in a[1:])
                r = _Value()
                for x in at:
                    if isinstance(x, _Value) and x is not r:
                        r = r.joined(x) if x.sums != r.sums or x.xs is not r.xs else r
                self.put(a[0], r)
            elif op == "v_mov_b32" and isinstance(self.val(a[1]), _Value):
                self.put(a[0], self.val(a[1]))
            elif op.startswith("v_mbcnt"):
                assert a[1] == "-1"
                self.put(a[0], np.minimum(lanes, 32) if "_lo_" in op else np.maximum(lanes - 32, 0) + self.val(a[2]))
            elif op in ("v_mad_u32_u24",):
                x, y, z = (self.val(q) for q in a[1:])
                assert (np.asarray(x) < 1 << 24).all() and y < 1 << 24
                self.put(a[0], x * y + z)
            elif op == "v_add_co_u32":
                r = np.asarray(self.val(a[2]), dtype=np.int64) + self.val(a[3])
                self.put(a[0], r)
                self.s["vcc"] = np.broadcast_to(r >> 32, 64)
            elif op == "v_addc_co_u32":
                self.put(a[0], np.asarray(self.val(a[2]), dtype=np.int64) + self.val(a[3]) + self.s["vcc"])
            else:
                f = {"v_mov_b32": lambda x: x, "v_add_u32": lambda x, y: x + y, "v_xor_b32": lambda x, y: x ^ y, "v_min_u32": np.minimum,
                     "v_and_b32": lambda x, y: x & y, "v_lshlrev_b32": lambda x, y: y << x, "v_lshrrev_b32": lambda x, y: y >> x,
                     "v_mul_lo_u32": lambda x, y: x * y, "v_mul_hi_u32": lambda x, y: x * y >> 32}.get(op)
                assert f or op in ("s_nop", "s_cbranch_scc1"), ln
                if f:
                    self.put(a[0], f(*(np.asarray(self.val(x), dtype=np.int64) for x in a[1:])))
        assert not any(q[0] == "lds" or q[0] == "scale" for q in self.queue)      # no load is on its way when the wave ends

    def put(self, d, x):
        n = int(d[1:])
        self.written_at[n] = -1
        if isinstance(x, _Value):
            self.held.pop(n & ~3, None)
            self.v[n] = x
            return
        if n < rows.ADDRW:
            # an address in scratch between tiles: only where the fragments are used up
            self.held.pop(n & ~3, None)
        self.v[n] = np.broadcast_to(np.asarray(x, dtype=np.int64) & U32, 64).copy()


@pytest.mark.parametrize("kind,save", [("i8", False), ("gated", False), ("gated", True)])
@pytest.mark.parametrize("mt,shape,tiles,pad,form", [
    (8, (300, 520, 256), [(0, 0), (1, 2), (0, 1), (1, 0)], 1, 0), (8, (513, 264, 768), [(2, 1), (0, 0)], 0, 10), (8, (256, 768, 256), [(0, 0), (0, 1), (0, 2)], 3, 4),
    (6, (200, 512, 512), [(0, 0), (0, 1), (1, 0)], 0, 10), (6, (193, 8, 256), [(1, 0)], 1, 0), (4, (129, 776, 256), [(1, 3), (0, 0), (0, 1), (1, 0)], 2, 4),
    (4, (1, 256, 1792), [(0, 0)], 0, 10)])
def test_loop_over_tiles(kind, save, mt, shape, tiles, pad, form):
    """Four waves in step from barrier to barrier: every load lies inside its operand and goes where nobody reads any more, every product takes
    the rows and bytes of its tile, stage and step from registers that have them, every sum is complete when it leaves, with the
    scales of its row and column (8 bits) or the gate's and the up projection's sum of one element (gated), and each element of the
    tiles is stored once, where it belongs; nothing outside."""
    M, N, _ = shape
    cols = 128 if kind == "gated" else 256
    if kind == "gated":
        tiles = [(tm, min(tn, (N - 1) // 128)) for tm, tn in tiles]
    text = [p for ln in rows.generate(mt, kind) for p in ln.split("\n")]
    lds = G._Lds()
    waves = [_Wave(kind, mt, w, text, lds, shape, tiles, pad, form, save) for w in range(4)]
    going = [w.run() for w in waves]
    while going:
        ends = [next(g, "end") for g in going]
        assert len(set(ends)) == 1
        if ends[0] == "end":
            break
        pending = np.zeros(len(lds.row), bool)
        for w in waves:
            for q in w.queue:
                if q[0] == "lds":
                    pending[q[1]] = True
        lds.visible = (lds.row >= 0) & ~pending
    want = {(m, n) for tm, tn in tiles for m in range(32 * mt * tm, min(32 * mt * (tm + 1), M)) for n in range(cols * tn, min(cols * (tn + 1), N), 8)}
    got = [k for w in waves for k in w.written]
    assert len(got) == len(want) and set(got) == want
    kept = [k for w in waves for k in w.saved]
    blocks = {(m // 16, n // 32) for m, n in want} if save else set()            # whole blocks, of those that hold anything
    assert len(kept) == len(set(kept)) and set(kept) == {(16 * i + r, 32 * j + c, up) for i, j in blocks for r in range(16) for c in range(0, 32, 4) for up in (False, True)}
    assert all(w.forms.get(t, "") == rows.FORMS[form >> 2 if t == len(tiles) - 1 else form & 3].strip() for w in waves if w.written for t in w.forms)


@pytest.mark.parametrize("mt", [8, 6, 4])
@pytest.mark.parametrize("kind", KINDS)
def test_wait_states(kind, mt):
    text = rows.generate(mt, kind)
    assert WS.too_close(text) == []
    # ... and their loads to LDS stay off the M0 write before them
    lines = [p for ln in text for p in ln.split("\n")]
    assert not any(ln.startswith("global_load_lds") and " m0," in lines[k - 1] for k, ln in enumerate(lines))


@pytest.mark.parametrize("file", ["gemm_i8", "gemm_gated"])
def test_kernels_do_not_spill(tmp_path, file):
    spec = importlib.util.spec_from_file_location("_flags", os.path.join(ROOT, "paper_2511_20426_amd", "_build.py"))
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)
    subprocess.run([sys.executable, os.path.join(build.CSRC, "gen_gemm_rows.py"), str(tmp_path / "gemm_rows_gfx950.inc")], check=True, capture_output=True)
    out = tmp_path / "out.s"
    subprocess.run([build.hipcc(), "-x", "hip", "-S", "--offload-device-only", os.path.join(build.CSRC, file + ".hip"), "-o", str(out), "-O3",
                    "-std=c++17", "--offload-arch=gfx950", "-I", os.path.join(ROOT, "include"), "-I", build.CSRC, "-I", str(tmp_path)] +
                   build.DEVICE_FLAGS + build.FILE_FLAGS.get(file + ".hip", []), check=True, capture_output=True)
    text = out.read_text()
    names = re.findall(r"\.name:\s*(\S*_kernel\S*)", text)
    spilled = [int(n) for n in re.findall(r"\.[sv]gpr_spill_count:\s*(\d+)", text)]
    assert len(names) >= 8 and len(spilled) == 2 * len(names) and not any(spilled), list(zip(names, spilled[::2], spilled[1::2]))
