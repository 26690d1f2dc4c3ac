"""The microscaled cache from its definition, in 64 bits (numpy): what the kernels are compared with."""
from __future__ import annotations

import numpy as np
import torch

from oracle import quoka_oracle as O
from paper_2602_08722_b200 import api

E_MIN, E_MAX = -64, 15


def element_values(fmt):
    """The value of every element code."""
    if fmt == api.KV_MXFP4:
        m = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
        return np.concatenate([m, -m])
    c = np.arange(128)
    e, f = c >> 3, c & 7
    m = np.where(e > 0, (8 + f) * 2.0 ** (e - 7.0 - 3), f * 2.0 ** (-6 - 3))
    m[127] = np.nan
    return np.concatenate([m, -m])


def quantise(x, fmt):
    """x (..., d) of finite or non-finite values -> (codes (..., d), scale bytes (..., d / 32))."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    most = 448.0 if fmt == api.KV_MXFP8 else 6.0
    finite = np.isfinite(blocks).all(-1)
    amax = np.where(finite, np.abs(np.where(np.isfinite(blocks), blocks, 0)).max(-1), 0.0)
    e = np.full(amax.shape, E_MIN)
    for cand in range(E_MIN, E_MAX):
        e = np.where(amax > most * 2.0 ** cand, cand + 1, e)
    y = np.where(finite[..., None], blocks, 0.0) * 2.0 ** -e[..., None].astype(np.float64)
    mags = element_values(fmt)[: 127 if fmt == api.KV_MXFP8 else 8]             # ascending; the index is the code
    a = np.minimum(np.abs(y), most)
    hi = np.searchsorted(mags, a)                                               # mags[hi - 1] < a <= mags[hi]
    lo = np.maximum(hi - 1, 0)
    down, up = a - mags[lo], mags[hi] - a
    code = np.where(down < up, lo, np.where(up < down, hi, np.where(lo % 2 == 0, lo, hi)))   # ties: the even fraction
    sign_bit = 128 if fmt == api.KV_MXFP8 else 8
    code = code + np.where(np.signbit(y), sign_bit, 0)
    code = np.where(finite[..., None], code, 0)
    scale = np.where(finite, e + 127, 255)
    return code.reshape(x.shape).astype(np.uint8), scale.astype(np.uint8)


def values(codes, scale, fmt):
    x = element_values(fmt)[codes].reshape(*codes.shape[:-1], -1, 32)
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return (x * s[..., None]).reshape(codes.shape)


def pack(codes, fmt):
    return codes if fmt == api.KV_MXFP8 else (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


class MxProblem:
    """One layer's microscaled cache on the device, filled from `inp` (synth.ChunkInputs) by the reference quantiser, and what it
    stands for in 64 bits (k64, v64: (b, n_KV, rows, d)).  layout: "bhtd", or "bthd" (head strides below row strides) with padding."""

    def __init__(self, inp, fmt, *, paged=False, max_ctx_len=None, impl=api.IMPL_AUTO, n_retain=16, kv_budget=0, budget_frac=0.0,
                 layout="bhtd", cached_norms=False, garbage=True, q_layout="bhcd", softmax_scale=0.0):
        self.inp, self.fmt = inp, fmt
        b, n_q, C, d = inp.q.shape
        n_kv = inp.k.shape[1]
        self.b, self.n_q, self.n_kv, self.C, self.d = b, n_q, n_kv, C, d
        self.max_ctx = int(inp.ctx_len.max()) if max_ctx_len is None else max_ctx_len
        rows = self.max_ctx + C + 3
        self.host = {}
        for name, x in (("k", inp.k), ("v", inp.v)):
            full = np.zeros((b, n_kv, rows, d))
            full[:, :, : x.shape[2]] = x.double().numpy()[:, :, :rows]
            codes, scale = quantise(full, fmt)
            for s in range(b):                        # beyond a sequence's rows the cache holds whatever it did, NaN blocks among it
                if garbage:
                    end = int(inp.ctx_len[s]) + C
                    codes[s, :, end:] = 0x7F if fmt == api.KV_MXFP8 else 7
                    scale[s, :, end:] = 255
            self.host[name] = (codes, scale)
        self.k64, self.v64 = (values(*self.host[n], fmt) for n in "kv")
        dev = "cuda"
        self.ctx_len = inp.ctx_len.to(dev)
        self.table = None
        if paged:
            need = [-(-(int(t) + C) // 64) for t in inp.ctx_len.tolist()]
            perm = np.random.default_rng(int(inp.ctx_len.sum())).permutation(sum(need) + 2)
            table = np.full((b, -(-(self.max_ctx + C) // 64)), -1, dtype=np.int32)
            off = 0
            for s, n in enumerate(need):
                table[s, :n] = perm[off:off + n]
                off += n
            self.table_host = table
            self.table = torch.from_numpy(table).to(dev)
        dev_t = {}
        for name in "kv":
            codes, scale = self.host[name]
            packed = pack(codes, fmt)
            if paged:
                pools = []
                for arr, fill in ((packed, 0x7F), (scale, 255)):
                    pool = np.full((len(perm), n_kv, 64, arr.shape[-1]), fill, dtype=np.uint8)
                    for s in range(b):
                        for i in range(need[s]):
                            n = min(64, rows - 64 * i)
                            pool[table[s, i], :, :n] = arr[s, :, 64 * i:64 * i + n]
                    pools.append(pool)
                packed, scale = pools
            dev_t[name] = (self._lay_out(torch.from_numpy(packed).to(dev), layout), torch.from_numpy(np.ascontiguousarray(scale)).to(dev))
        (self.k, self.k_scale), (self.v, self.v_scale) = dev_t["k"], dev_t["v"]
        self.q = inp.q.to(dev)
        if q_layout == "bchd":
            self.q = self.q.transpose(1, 2).contiguous().transpose(1, 2)
        self.out = torch.full_like(self.q, 7.0)
        self.lse = torch.full((b, n_q, C), 7.0, device=dev)
        self.p = api.make_params(self.q, self.k, self.out, self.ctx_len, n_retain=n_retain, kv_budget=kv_budget, budget_frac=budget_frac,
                                 max_ctx_len=self.max_ctx, block_table=self.table, impl=impl, kv_format=fmt, softmax_scale=softmax_scale)
        self.mx = api.make_mx_cache(fmt, self.k_scale, self.v_scale)
        self.norms = None
        if cached_norms:
            with np.errstate(invalid="ignore"):
                inv = 1.0 / np.maximum(np.sqrt((self.k64 ** 2).sum(-1)), 1e-12)
            if paged:
                pool = np.full((len(perm), n_kv, 64), np.nan)
                for s in range(b):
                    for i in range(need[s]):
                        n = min(64, rows - 64 * i)
                        pool[table[s, i], :, :n] = inv[s, :, 64 * i:64 * i + n]
                inv = pool
            self.norms = torch.from_numpy(inv).float().to(dev)
            self.p.k_inv_norm = self.norms.data_ptr()
        self.ws = api.alloc_workspace(self.p, mx=self.mx)
        self.cap = api.quoka_kv_budget_cap(self.p)

    @staticmethod
    def _lay_out(t, layout):
        if layout == "bhtd":
            return t
        b, h, r, n = t.shape                          # rows 32 bytes apart from each other, heads next to each other
        room = torch.full((b, r, h, n + 32), 0x55, dtype=torch.uint8, device=t.device)
        view = room[..., :n].transpose(1, 2)
        view.copy_(t)
        return view

    def listed(self, seed=0, counts=None):
        """A random list of rows per (sequence, KV head), on the device, and on the host as index arrays."""
        r = np.random.default_rng(seed)
        idx = np.full((self.b, self.n_kv, self.cap), -1, dtype=np.int32)
        cnt = []
        for s in range(self.b):
            T = int(self.inp.ctx_len[s])
            n = min(self.cap, T) if counts is None else counts[s]
            cnt.append(n)
            for h in range(self.n_kv):
                idx[s, h, :n] = np.sort(r.permutation(T)[:n])
        self.idx_host, self.cnt_host = idx, cnt
        return torch.from_numpy(idx).cuda(), torch.tensor(cnt, dtype=torch.int32, device="cuda")

    def reference(self, s, rows=None, use_list=False):
        """(out, lse) of sequence s in 64 bits; with `rows` = (heads, rows) the outputs of these."""
        T = int(self.inp.ctx_len[s])
        q = self.inp.q[s].double().numpy()
        k, v = self.k64[s, :, :T + self.C], self.v64[s, :, :T + self.C]
        lists = [self.idx_host[s, h, :self.cnt_host[s]] if use_list else np.arange(T) for h in range(self.n_kv)]
        if rows is not None:
            return O.sparse_attention_rows(q, k, v, T, lists, *rows), None
        return O.sparse_attention(q, k, v, T, lists)
