"""Which kernels a call over a microscaled cache runs (the launch log of a process of its own)."""
import os
import re
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = """
import torch
from paper_2602_08722_b200 import api, synth
from tests import mx_reference as R
inp = synth.make_chunk_inputs(1, 1, {n_q}, {n_kv}, {d}, [{T}], {C}, "bf16")
P = R.MxProblem(inp, api.KV_MXFP8, kv_budget={budget}, n_retain={n_retain})
args = P.listed(5)
if {entry!r} == "score":
    qbar = torch.zeros(1, {n_kv}, min({n_retain}, {C}), {d}, dtype=torch.bfloat16, device="cuda")
    api.quoka_score_keys_mx(P.p, P.mx, qbar, P.k, torch.empty(1, {n_kv}, {T}, device="cuda"), P.ws)
else:
    if {entry!r} == "listed":
        api.quoka_sparse_attn_mx(P.p, P.mx, P.q, P.k, P.v, *args, P.out, None, P.ws)
    elif {entry!r} == "dense":
        api.quoka_dense_chunk_attn_mx(P.p, P.mx, P.q, P.k, P.v, P.out, None, P.ws)
    else:
        api.quoka_prefill_chunk_mx(P.p, P.mx, P.q, P.k, P.v, P.out, None, None, P.ws)
torch.cuda.synchronize()
"""


@pytest.mark.parametrize("entry,n_q,n_kv,d,C,T,n_retain,runs,not_runs", [
    ("listed", 8, 1, 64, 300, 400, 16, ["unpack_rows_mx", "attn_tc(_pair)?_unpacked"], ["attn_tc(_pair)?_mx"]),
    ("fused", 8, 1, 128, 300, 400, 16, ["score_keys_mx_tc", "unpack_rows_mx", "attn_tc(_pair)?_unpacked"], ["attn_tc(_pair)?_mx"]),
    ("dense", 8, 1, 128, 300, 400, 16, ["attn_tc(_pair)?_mx"], ["unpack_rows_mx"]),
    ("dense", 16, 1, 128, 520, 400, 16, ["unpack_rows_mx", "attn_tc(_pair)?_unpacked"], ["attn_tc(_pair)?_mx"]),
    ("dense", 8, 1, 64, 300, 400, 16, ["unpack_rows_mx", "attn_tc(_pair)?_unpacked"], ["attn_tc(_pair)?_mx"]),
    ("listed", 8, 2, 128, 1, 400, 1, ["decode_mx"], ["attn_tc.*"]),
    ("score", 8, 2, 128, 8, 400, 8, ["score_few_mx"], ["score_keys_mx_tc"]), ("score", 8, 2, 128, 9, 400, 9, ["score_keys_mx_tc"], ["score_few_mx"])])
def test_kernels(entry, n_q, n_kv, d, C, T, n_retain, runs, not_runs):
    code = CODE.format(entry=entry, n_q=n_q, n_kv=n_kv, d=d, C=C, T=T, n_retain=n_retain, budget=200)
    run = subprocess.run([sys.executable, "-c", code], cwd=ROOT, env=dict(os.environ, QUOKA_LOG="1"), capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr
    ran = re.findall(r"\[quoka\] (\w+) ", run.stderr)

    def has(pattern):
        return any(re.fullmatch(pattern, name) for name in ran)
    assert all(map(has, runs)) and not any(map(has, not_runs)), ran
