"""The first use of a call of ssd_step.h on a device sets up all of its kernels: captures with other types and sizes in a fresh process."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import sys
sys.path.insert(0, sys.argv[1])
import torch
import paper_2309_08168_gb300 as ssd

gen = torch.Generator().manual_seed(1)


def normal(t, *shape, std=1.0):
    return (std * torch.randn(*shape, generator=gen)).to(t).cuda()


def layer(t, n):
    e, d, f, k = 4, 64, 40, 2
    x, w, m = normal(t, n, d), normal(t, e, d), ssd.MoeWeights(*(normal(t, *s, std=0.125) for s in ((e, f, d), (e, f, d), (e, d, f))))
    ids, weights, out = torch.zeros(n, k, dtype=torch.int32, device="cuda"), torch.zeros(n, k, device="cuda"), torch.zeros(n, d, dtype=t, device="cuda")
    ws = torch.zeros(ssd.ssd_moe_workspace(m, n, k), dtype=torch.uint8, device="cuda")

    def run(s):
        ssd.ssd_moe_route(x, w, ids, weights, cuda_stream=s)
        ssd.ssd_moe_mlp(m, x, ids, weights, out, ws, cuda_stream=s)
    return run, [ids, weights, out]


def heads(t, n):
    c = torch.float16 if t is torch.float32 else t
    q, k, v, out = normal(t, n, 4, 64), normal(t, n, 1, 64), normal(t, n, 1, 64), torch.zeros(n, 4, 64, dtype=t, device="cuda")
    cache = [torch.zeros(1, n // 16 + 1, 1, 16, 64, dtype=c, device="cuda") for _ in range(2)]
    kv, rope, rows = ssd.PagedKV(*cache), ssd.ssd_rope_init(64), torch.arange(n, dtype=torch.int32, device="cuda")

    def run(s):
        ssd.ssd_norm_rope_kv(kv, 0, rope, q, k, v, rows, rows, out, cuda_stream=s)
    return run, [out, *cache]


def logits(t, n, bias, lead):
    x, v = normal(t, n, 1003), 1003 - lead
    b = normal(torch.float32, 1, v) if bias else None
    allowed = torch.full((n, (v + 31) // 32), 0x5f5f5f5f, dtype=torch.int32, device="cuda") if bias else None
    rules = ssd.LogitRules(v, n, bias=b, allowed=allowed)
    tokens, logprob, out = torch.zeros(n, 2, dtype=torch.int32, device="cuda"), torch.zeros(n, 2, device="cuda"), torch.zeros(n, v, dtype=t, device="cuda")

    def run(s):
        ssd.ssd_logits_choose(rules, x[:, lead:], tokens, logprob, None, s)
        ssd.ssd_logits_adjust(rules, x[:, lead:], out, s)
    return run, [tokens, logprob, out]


f32, f16, bf16 = torch.float32, torch.float16, torch.bfloat16
for run, _ in (layer(bf16, 1), heads(bf16, 1), logits(bf16, 1, False, 0)):
    run(torch.cuda.current_stream().cuda_stream)
torch.cuda.synchronize()
cases = [layer(t, n) for t in (bf16, f16) for n in (9, 40)] + [heads(t, n) for t in (f32, f16, bf16) for n in (3, 2500)]
cases += [logits(t, n, bias, lead) for t in (f32, f16, bf16) for n in (2, 700) for bias in (False, True) for lead in (0, 3)]
torch.cuda.synchronize()
for i, (run, outs) in enumerate(cases):
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(torch.cuda.current_stream().cuda_stream)
    g.replay()
    torch.cuda.synchronize()
    got = [o.clone() for o in outs]
    for o in outs:
        o.zero_()
    run(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, outs)) and all(bool(a.float().abs().sum() > 0) for a in got), i
print("as eager:", len(cases))
"""


def test_one_use_prepares_all_captures():
    r = subprocess.run([sys.executable, "-c", CODE, ROOT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "as eager: 34", (r.returncode, r.stdout[-500:], r.stderr[-3000:])
