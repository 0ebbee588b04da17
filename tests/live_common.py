"""Plain 64-bit reference of the live-cache calls, and the batches their tests run on.  The reference shares no code with
the library: pages are built and taken apart here with numpy, attention is a float64 loop over sequences and heads."""
from __future__ import annotations

from dataclasses import dataclass
from typing import List, Optional

import numpy as np
import torch

BITS = {1: (8, 8), 2: (8, 4), 3: (4, 4)}          # K and V bits by tag
F16, BF16 = torch.float16, torch.bfloat16


def quantise64(x: np.ndarray, bits: int, group: int):
    """float64 [..., D] -> integer codes [..., D] and fp16 scales [..., D / group].  The quotient amax / qmax of a value
    with at most 11 significant bits is 2^-19 or more away from an fp16 rounding border, so one rounding from 64 bits
    gives the same scale as fp32 division followed by rounding."""
    top = 2 ** (bits - 1) - 1
    g = x.reshape(*x.shape[:-1], -1, group)
    with np.errstate(over="ignore"):
        s = (np.abs(g).max(-1) / top).astype(np.float16)
    sd = s.astype(np.float64)
    ok = (sd > 0) & np.isfinite(sd)
    q = np.where(ok[..., None], np.rint(g / np.where(ok, sd, 1.0)[..., None]), 0.0)
    return np.clip(q, -top, top).astype(np.int64).reshape(x.shape), s


def pack(q: np.ndarray, bits: int) -> np.ndarray:
    flat = q.reshape(-1)
    if bits == 8:
        return flat.astype(np.int8).view(np.uint8)
    return ((flat[0::2] & 15) | ((flat[1::2] & 15) << 4)).astype(np.uint8)


def unpack(b: np.ndarray, bits: int) -> np.ndarray:
    if bits == 8:
        return b.view(np.int8).astype(np.int64)
    n = np.stack([b & 15, b >> 4], -1).reshape(-1).astype(np.int64)
    return np.where(n > 7, n - 16, n)


@dataclass
class Layout:
    tag: int
    H: int
    D: int
    P: int
    G: int

    def sections(self):
        e = self.P * self.H * self.D
        kb, vb = BITS[self.tag]
        return [e * kb // 8, 2 * e // self.G, e * vb // 8, 2 * e // self.G]

    def page_bytes(self):
        return -(-sum(self.sections()) // 16) * 16

    def split(self, page: np.ndarray):
        """(codes, scales) of K and of V as views of a page's bytes."""
        out, at = [], 0
        for n in self.sections():
            out.append(page[at:at + n])
            at += n
        return out

    def values(self, page: np.ndarray):
        """K and V of a page as float64 [P][H][D]."""
        kc, ks, vc, vs = self.split(page)
        out = []
        for codes, scales, bits in ((kc, ks, BITS[self.tag][0]), (vc, vs, BITS[self.tag][1])):
            s = np.frombuffer(scales.tobytes(), np.float16).astype(np.float64)
            with np.errstate(invalid="ignore"):
                out.append((unpack(codes, bits).reshape(-1, self.G) * s[:, None]).reshape(self.P, self.H, self.D))
        return out

    def put(self, page: np.ndarray, slot: int, k: np.ndarray, v: np.ndarray):
        """Quantises one token's K and V (float64 [H][D]) into a slot.  Codes of a slot are whole bytes (D is even)."""
        kc, ks, vc, vs = self.split(page)
        for x, codes, scales, bits in ((k, kc, ks, BITS[self.tag][0]), (v, vc, vs, BITS[self.tag][1])):
            q, s = quantise64(x, bits, self.G)
            n = self.H * self.D * bits // 8
            codes[slot * n:(slot + 1) * n] = pack(q, bits)
            m = 2 * self.H * self.D // self.G
            scales[slot * m:(slot + 1) * m] = np.frombuffer(s.tobytes(), np.uint8)


@dataclass
class Case:
    """A ragged batch: kv_len and rows per sequence, and the positions (None: the last ones)."""
    kv: List[int]
    rows: List[int]
    pos: Optional[List[List[int]]] = None

    def positions(self):
        if self.pos is not None:
            return [list(p) for p in self.pos]
        return [[t - r + i for i in range(r)] for t, r in zip(self.kv, self.rows)]


def build_tables(case: Case, P: int, rng, spare: int = 3):
    per = max(1, max(-(-t // P) for t in case.kv)) if case.kv else 1
    n_pages = len(case.kv) * per + spare
    table = rng.permutation(n_pages)[:len(case.kv) * per].reshape(len(case.kv), per).astype(np.int32)
    return table, n_pages


def device_batch(pk, case: Case, table: np.ndarray, dev, n_rows=None, max_rows=None, max_kv=None):
    start = np.concatenate([[0], np.cumsum(case.rows)]).astype(np.int32)
    keep = {"start": torch.from_numpy(start).to(dev), "kv": torch.tensor(case.kv, dtype=torch.int32, device=dev),
            "table": torch.from_numpy(np.ascontiguousarray(table)).to(dev), "pos": None}
    n = int(start[-1]) if n_rows is None else n_rows
    if case.pos is not None:
        flat = [p for s in case.pos for p in s] + [0] * (n - int(start[-1]))
        keep["pos"] = torch.tensor(flat, dtype=torch.int32, device=dev)
    b = pk.make_batch(row_start=keep["start"], kv_len=keep["kv"], block_table=keep["table"], n_rows=n,
                      max_rows=max(case.rows + [0]) if max_rows is None else max_rows,
                      max_kv_len=max(case.kv + [0]) if max_kv is None else max_kv, pos=keep["pos"])
    return b, keep


def random_rows(rng, n, H, D, dtype, outliers=True):
    x = rng.standard_normal((n, H, D))
    if outliers and D >= 16:
        x[..., rng.permutation(D)[:max(1, D // 20)]] *= 10
    return torch.from_numpy(x).to(dtype)


def attention64(q, k_of, v_of, case: Case, share: int, scale: float, window: int, sinks: int, out_type, bf16_pool: bool,
                k_rounding: float = 2.0 ** -11):
    """q float64 [n][Hq][D]; k_of(b), v_of(b): float64 [kv][H][D] of a sequence.  Returns (out, tol).

    tol is an elementwise bound on what the library may be off, from its number formats alone:
      the result's rounding                          u_out |o|
      the weights as 16-bit numbers                  u_p sum p|v|       (u_p 2^-8 over bf16 pages, 2^-11 else)
      quantised values as fp16 operands              2^-11 sum p|v|     and logits off by d = k_rounding scale max_j sum |q||k|,
                                                     which change a weight by a factor within e^(2d)
      fp32 sums (and exp2, 2^-22) over D, then the tokens in pieces: (D + 64) 2^-23 on the logits' terms likewise
      weights below fp16's normal range              n 2^-24 max|v|
    """
    u_out = torch.finfo(out_type).eps / 2
    n, Hq, D = q.shape
    out, tol = np.zeros((n, Hq, D)), np.zeros((n, Hq, D))
    r = 0
    for b, (t, positions) in enumerate(zip(case.kv, case.positions())):
        R = len(positions)
        if R == 0:
            continue
        K, V = k_of(b), v_of(b)
        j, p = np.arange(t)[None], np.array(positions)[:, None]
        see = (j <= p) & ((window == 0) | (p - j < window) | (j < sinks))
        some = see.any(0)                                  # what no row sees may hold anything
        K, V, see = K[some], V[some], see[:, some]
        live = see.any(1)
        if live.any():
            for h in range(Hq):
                kk, vv, qq = K[:, h // share], V[:, h // share], q[r:r + R, h]
                x = np.where(see, qq @ kk.T * scale, -np.inf)
                w = np.exp(x - np.where(live, x.max(1), 0.0)[:, None])
                w /= np.where(live, w.sum(1), 1.0)[:, None]
                o, a = w @ vv, w @ np.abs(vv)
                big = np.abs(scale) * np.where(see, np.abs(qq) @ np.abs(kk).T, 0.0).max(1)[:, None]
                d = ((0.0 if bf16_pool else k_rounding) + (D + 64) * 2.0 ** -23) * big
                u = (2.0 ** -8 if bf16_pool else 2.0 ** -11 + 2.0 ** -11) + np.expm1(2 * d) + 2.0 ** -18
                floor = see.sum(1)[:, None] * 2.0 ** -24 * np.abs(vv).max()
                out[r:r + R, h] = o
                tol[r:r + R, h] = u_out * np.abs(o) + (1 + u_out) * (u * a + floor) + (2.0 ** -25 if out_type == F16 else 1e-30)
        r += R
    return out, tol
