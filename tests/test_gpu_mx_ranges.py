"""Keys, values and queries that span the range of the microscaled cache's scales, against the definition in 64 bits.

Tolerances.  A logit is a sum of at most 128 exact products in fp32 (at most 130 roundings or truncations of a partial sum, 2^-23 of the
sum of magnitudes each), times a scale (four roundings of the logit), and its exponential is off by 2^-21: with d_j for all of this, the
weight of key j is off by d_j of itself and the sum of weights by the mean of d_j.  Weights are rounded to bf16 at worst, by half a step, 2^-8 of
the weight (8 bits: finfo(bfloat16).eps / 2), and the sum may be of weights before that, 2^-8 more; the fp32 sums over n keys add
n 2^-23, the rounding of the output to bf16 2^-8 of it.
So every bound is on the weighted magnitudes sum_j p_j |v_j| of the row itself: a value of no weight, or that a row does not see, adds nothing.
"""
import numpy as np
import pytest
import torch

from paper_2602_08722_b200 import api, synth
from tests import mx_reference as R
from tests import parity as PA

pytestmark = pytest.mark.gpu
FORMATS = [api.KV_MXFP8, api.KV_MXFP4]


def attention64(q, k, v, T, scale):
    """(out, bound) of one head: q (C, d), k and v (T + C, d)."""
    logit = q @ k.T * scale
    hidden = np.arange(k.shape[0])[None] > T + np.arange(q.shape[0])[:, None]
    logit[hidden] = -np.inf
    p = np.exp(logit - logit.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    d = 130 * 2.0 ** -23 * scale * (np.abs(q) @ np.abs(k).T) + 4 * 2.0 ** -24 * np.abs(np.where(hidden, 0, logit)) + 2.0 ** -21
    mag = p @ np.abs(v)
    out = p @ v
    off = (p * d).sum(-1, keepdims=True)
    bound = (p * d) @ np.abs(v) + mag * (off + 2.0 ** -7 + k.shape[0] * 2.0 ** -23) + np.abs(out) * 2.0 ** -8
    return out, bound


def push(inp, t, logits):
    """Column 0 of the queries is 8 and of key t what gives the logits (others as small as the noise of the other columns)."""
    d = inp.q.shape[-1]
    inp.q[..., 0] = 8
    inp.k[:, :, t, 0] = (logits * d ** 0.5 / 8).bfloat16()


def problem(kind, n_q, n_kv, d, T, C, seed):
    """One sequence whose keys, values or queries span more than fp16 does."""
    g = torch.Generator().manual_seed(seed)
    inp = synth.make_chunk_inputs(seed, 1, n_q, n_kv, d, [T], C, "bf16")
    for x, size in ((inp.q, 0.3), (inp.k, 0.3), (inp.v, 1.0)):
        x.copy_((torch.randn(x.shape, generator=g) * size).bfloat16())
    everyone = torch.arange(T + C)
    if kind == "large values of little weight":                 # what they add is most of the output
        push(inp, everyone, torch.randn(T + C, generator=g) * 0.5)
        push(inp, torch.tensor([10]), torch.tensor([23.0]))       # its weight is 2^31 to 2^35 times that of the others
        inp.v *= 2.0 ** 10
        inp.v[:, :, 10] *= 2.0 ** -34
    elif kind == "a large value of no weight":
        push(inp, everyone, torch.zeros(T + C))
        push(inp, torch.tensor([T // 2]), torch.tensor([-60.0]))
        inp.v *= 2.0 ** -32
        inp.v[:, :, T // 2] *= 2.0 ** 46
    elif kind == "the smallest values beside the largest":
        push(inp, everyone, torch.zeros(T + C))
        push(inp, torch.tensor([T - 3]), torch.tensor([-150.0]))
        inp.v *= 2.0 ** -63
        inp.v[:, :, T - 3] *= 2.0 ** 77
    elif kind == "large values in rows that others do not see":
        inp.v *= 2.0 ** -30
        inp.v[:, :, T + 1:] *= 2.0 ** 44
    elif kind == "small blocks of keys":                        # queries are zero on the large block
        inp.k[..., :32] *= 2.0 ** 15
        inp.k[..., 32:] *= 2.0 ** -24
        inp.q[..., :32] = 0
        inp.q[..., 32:] *= 2.0 ** 26
    elif kind == "a block of zeros in every key":
        inp.k[..., -32:] = 0
        inp.k *= 4
    elif kind == "queries of a wide range":
        inp.k[..., 3] = 0
        inp.q *= 10
        inp.q[..., 3] = 2.0 ** 60
    elif kind == "everything":
        e = torch.randint(-40, 12, (1, n_kv, T + C, d // 32), generator=g).double().repeat_interleave(32, -1)
        inp.v.copy_((inp.v.double() * 2.0 ** e).bfloat16())
        e = torch.randint(-30, 3, (1, n_kv, T + C, d // 32), generator=g).double().repeat_interleave(32, -1)
        inp.k.copy_((inp.k.double() * 2.0 ** e).bfloat16())
        inp.q *= 4
    return inp


KINDS = ["large values of little weight", "a large value of no weight", "the smallest values beside the largest",
         "large values in rows that others do not see", "small blocks of keys", "a block of zeros in every key",
         "queries of a wide range", "everything"]
SHAPES = [(4, 1, 128, 1), (8, 2, 128, 4), (8, 1, 64, 5), (2, 1, 64, 3), (6, 2, 64, 7), (4, 1, 128, 70), (8, 1, 64, 270)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T", [600, 5000])
@pytest.mark.parametrize("n_q,n_kv,d,C", SHAPES)
def test_attention(kind, fmt, T, n_q, n_kv, d, C):
    P = R.MxProblem(problem(kind, n_q, n_kv, d, T, C, 61), fmt, kv_budget=T, max_ctx_len=T)
    P.listed(3)                                               # the whole cache
    outs = {}
    api.quoka_dense_chunk_attn_mx(P.p, P.mx, P.q, P.k, P.v, P.out, None, P.ws)
    outs["dense"] = PA.f64(P.out[0])
    k_idx, k_cnt = torch.from_numpy(P.idx_host).cuda(), torch.tensor(P.cnt_host, dtype=torch.int32, device="cuda")
    api.quoka_sparse_attn_mx(P.p, P.mx, P.q, P.k, P.v, k_idx, k_cnt, P.out, None, P.ws)
    outs["listed"] = PA.f64(P.out[0])
    assert api.quoka_last_device_status(P.ws) == 0
    q = P.inp.q[0].double().numpy()
    for h in range(n_q):
        kv = h // (n_q // n_kv)
        want, bound = attention64(q[h], P.k64[0, kv, :T + C], P.v64[0, kv, :T + C], T, d ** -0.5)
        for name, got in outs.items():
            worst = (np.abs(got[h] - want) / bound).max()
            assert worst <= 1, (name, h, worst)


@pytest.mark.parametrize("kind", ["small blocks of keys", "a block of zeros in every key", "queries of a wide range", "everything"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("norms", [False, True])
@pytest.mark.parametrize("n_kv,d,T,N", [(2, 128, 600, 1), (1, 64, 777, 1), (1, 128, 300, 5), (2, 64, 300, 8), (1, 128, 700, 20), (1, 64, 200, 70)])
def test_scores(kind, fmt, norms, n_kv, d, T, N):
    """Products are exact and so is a square; 130 roundings of a sum as above, of the squares 2^-23 each as well, a root, a division."""
    inp = problem(kind, n_kv, n_kv, d, T, N, 62)
    P = R.MxProblem(inp, fmt, n_retain=N, kv_budget=8, cached_norms=norms, max_ctx_len=T)
    qbar = inp.q.clone()                                      # (b, n_kv, N, d): a head per KV head
    scores = torch.full((1, n_kv, T), 7.0, device="cuda")
    api.quoka_score_keys_mx(P.p, P.mx, qbar.cuda(), P.k, scores, P.ws)
    assert api.quoka_last_device_status(P.ws) == 0
    for h in range(n_kv):
        qb, k = qbar[0, h].double().numpy(), P.k64[0, h, :T]
        norm = np.maximum(np.sqrt((k ** 2).sum(-1)), 1e-12)
        want = (qb @ k.T / norm).max(0)
        bound = (130 * 2.0 ** -23 * (np.abs(qb) @ np.abs(k).T) / norm).max(0) + 140 * 2.0 ** -23 * np.abs(want)
        worst = (np.abs(PA.f64(scores[0, h]) - want) / bound).max()
        assert worst <= 1, (h, worst)
