"""The 8-bit attention of a batch whose cu_nodes run backwards, so that sequences overlap and
make more work items than the nodes alone would: the call reports the malformed tree, and
nodes that belong to one well-formed sequence only keep their outputs."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

# cu_nodes, contexts, page, Hq, Hkv, D, nodes of one sequence only: more items than SMs,
# pages, and a batch small enough to be planned in chunks
CASES = [
    ([0, 100, 50, 150], [300, 0, 10], 0, 128, 32, 64, [(0, 0, 50), (2, 100, 150)]),
    ([0, 100, 50, 150], [300, 0, 10], 16, 256, 32, 128, [(0, 0, 50), (2, 100, 150)]),
    ([x for k in range(7) for x in (k, 128 + k)], [200] * 13, 0, 32, 8, 128,
     [(0, 0, 1), (12, 133, 134)]),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_overlapping_sequences(case):
    from paper_2609_02897_gb300 import asd, asd8
    cu, ctx, page, Hq, Hkv, D, unique = CASES[case]
    B, T, G, cap = len(cu) - 1, cu[-1], Hq // Hkv, 512
    gen = torch.Generator(device="cuda").manual_seed(case)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)
    q, tree_k, tree_v = normal(T, Hq, D), normal(T, Hkv, D), normal(T, Hkv, D)
    i32, per = torch.int32, cap // page if page else 0
    pages = B * per
    shape = (pages, Hkv, page, D) if page else (B, Hkv, cap, D)
    k16, v16 = normal(*shape), normal(*shape)
    table = torch.randperm(pages, generator=gen, device="cuda").view(B, per).int() if page else None
    dims = asd.make_dims(B, Hq, Hkv, D, 64, 64, asd.ASD_BF16, page, cap, pages, 128, 128)
    lens = torch.tensor(ctx, dtype=i32, device="cuda")
    parent = torch.zeros(T, dtype=i32)
    parent[cu[::2]] = -1                       # every well-formed sequence is a star
    cache, ws = asd8.Cache8(dims), asd8.alloc_workspace(dims, T).zero_()
    asd8.asd8_kv_quantize(dims, k16, v16, table, lens, cache, ws)
    out = torch.full((T, Hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    asd8.asd8_tree_attention(dims, q, cache, table, lens, tree_k, tree_v, parent.cuda(),
                             torch.tensor(cu, dtype=i32, device="cuda"), out, ws)
    assert asd.asd_get_device_status(ws) == 3
    k8, v8 = cache.values("k").double(), cache.values("v").double()
    for b, lo, hi in unique:
        for h in range(Hkv):
            def rows(x):
                return (x[table[b].long(), h].reshape(-1, D) if page else x[b, h])[:ctx[b]]
            for i in range(lo, hi):
                see = [cu[b]] + ([i] if i != cu[b] else [])
                k = torch.cat([rows(k8), tree_k[see, h].double()])
                v = torch.cat([rows(v8), tree_v[see, h].double()])
                p = (q[i, h * G:(h + 1) * G].double() @ k.T / math.sqrt(D)).softmax(1)
                err = (out[i, h * G:(h + 1) * G].double() - p @ v).abs()
                # the output's rounding, and those of the weights and scores (2^-8 each); few
                # of the weights are far below the largest: 2^-16 of it for each of 32 keys
                tol = 2.0 ** -8 * (p @ v).abs() + 2.0 ** -7 * (p @ v.abs()) + 2.0 ** -11 * v.abs().amax()
                assert (err <= tol).all(), (b, i, h)
