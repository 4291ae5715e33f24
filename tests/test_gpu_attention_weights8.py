"""Small softmax weights of the tree attention over the 8-bit cache: a token that takes most
of a row's weight in front of a long context, and V blocks whose scales lie far apart, must
not cost the output what the other tokens add.  Against float64 on the values that the
cache's bytes stand for."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

B16, F64 = torch.bfloat16, torch.float64


class Call:
    """Chains of `nodes` drafted tokens behind contexts `ctx`, pages of the pool in order.
    Scores of the context are N(0, spread); V has a mean of 1 and a spread of 0.5."""

    def __init__(self, seed, nodes, ctx, Hq, Hkv, D, page, spread=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.nodes, self.ctx, self.Hq, self.Hkv, self.D, self.page = nodes, ctx, Hq, Hkv, D, page
        T, B = sum(nodes), len(nodes)

        def normal(*shape):
            return torch.randn(*shape, generator=g, device="cuda")
        self.first, rows = [], 0                    # a sequence's slots follow each other
        for c in ctx:
            self.first.append(rows)
            rows += -(-c // page) * page
        self.num_pages = rows // page + 1
        self.k = normal(rows + page, Hkv, D) * spread
        self.v = 1 + 0.5 * normal(rows + page, Hkv, D)
        self.k[..., 0] = 0
        self.q = normal(T, Hq, D)
        self.q[..., 0] = 8.0
        self.tree_k, self.tree_v = normal(T, Hkv, D) * spread, 1 + 0.5 * normal(T, Hkv, D)
        self.tree_k[..., 0] = 0
        per = max(-(-c // page) for c in ctx) + -(-max(nodes) // page)
        self.table = torch.zeros(B, per, dtype=torch.int32)
        for b, c in enumerate(ctx):
            n = -(-c // page)
            self.table[b, :n] = self.first[b] // page + torch.arange(n, dtype=torch.int32)
        self.cap = per * page

    def score(self, b, lo, hi, x):
        """Adds x nats to the scores of positions lo .. hi - 1 of sequence b, all heads."""
        self.k[self.first[b] + lo:self.first[b] + hi, :, 0] = x * math.sqrt(self.D) / 8.0

    def dominant(self, b, weight, spread=1.0):
        """Position 0 takes about `weight` of every row, and holds a small V."""
        n = self.ctx[b]
        self.k[self.first[b], :, 1:] = 0
        self.score(b, 0, 1, math.log(weight / (1 - weight) * n) + spread * spread / 2)
        self.v[self.first[b]] *= 0.01

    def run(self):
        from paper_2609_02897_gb300 import asd, asd8
        pool = [x.view(self.num_pages, self.page, self.Hkv, self.D).transpose(1, 2).contiguous().to(B16)
                for x in (self.k, self.v)]
        dims = asd.make_dims(len(self.nodes), self.Hq, self.Hkv, self.D, 64, 64, asd.ASD_BF16, self.page,
                             self.cap, self.num_pages, max(self.nodes), max(self.nodes))
        T, i32 = sum(self.nodes), torch.int32
        cache, ws = asd8.Cache8(dims), asd8.alloc_workspace(dims, T)
        table, ctx = self.table.cuda(), torch.tensor(self.ctx, dtype=i32, device="cuda")
        asd8.asd8_kv_quantize(dims, *pool, table, ctx, cache, ws)
        parent = torch.cat([torch.arange(n, dtype=i32) - 1 for n in self.nodes]).cuda()
        cu = torch.tensor([0] + self.nodes).cumsum(0).to(i32).cuda()
        self.q16, self.tk16, self.tv16 = (x.to(B16) for x in (self.q, self.tree_k, self.tree_v))
        out = torch.full((T, self.Hq, self.D), float("nan"), dtype=B16, device="cuda")
        asd8.asd8_tree_attention(dims, self.q16, cache, table, ctx, self.tk16, self.tv16, parent, cu, out, ws)
        assert asd.asd_get_device_status(ws) == 0
        flat = [cache.values(w).transpose(1, 2).reshape(-1, self.Hkv, self.D).to(F64) for w in ("k", "v")]
        step = torch.ldexp(torch.ones_like(cache.v_exp, dtype=F64), cache.v_exp.int() - 127)
        step = step.repeat_interleave(cache.block, 2).transpose(1, 2).reshape(-1, self.Hkv)
        return out, flat[0], flat[1], step

    def check(self, seqs, most):
        """Every row of sequences `seqs`: each element within what the call may round, and
        the norm of a sequence's error within `most` of that of sum p |V|, which the roundings
        of weights are relative to (the output, where V has one sign).  What may round:
          the output, half a step of bf16: 2^-8 of it;
          a weight as the P.V product holds it: 2^-8 of it, or, in the context, 2^-16 of the
          largest product of a weight and a V scale among the 32 positions it is in;
          the scores (q's terms, fp32 sums), which moves a weight by less than 2^-8 of it."""
        out, k, v, step = self.run()
        G, t0 = self.Hq // self.Hkv, 0
        for b, n in enumerate(self.nodes):
            if b in seqs:
                at, c = slice(self.first[b], self.first[b] + self.ctx[b]), self.ctx[b]
                err2 = w2 = 0.0
                for h in range(self.Hkv):
                    kk = torch.cat([k[at, h], self.tk16[t0:t0 + n, h].to(F64)])
                    vv = torch.cat([v[at, h], self.tv16[t0:t0 + n, h].to(F64)])
                    q = self.q16[t0:t0 + n, h * G:h * G + G].to(F64)
                    x = torch.einsum("ngd,kd->ngk", q, kk) / math.sqrt(self.D)
                    see = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
                    x[:, :, c:] = x[:, :, c:].masked_fill(~see[:, None], -math.inf)
                    p = x.softmax(-1)
                    o, w = p @ vv, p @ vv.abs()
                    # a group's largest weight times scale, and its |V| in units of their scales
                    pad = -c % 32
                    ps = torch.nn.functional.pad(p[..., :c] * step[at, h], (0, pad)).unflatten(-1, (-1, 32))
                    vs = torch.nn.functional.pad(v[at, h].abs() / step[at, h, None], (0, 0, 0, pad))
                    few = ps.amax(-1) @ vs.unflatten(0, (-1, 32)).sum(1)
                    got = out[t0:t0 + n, h * G:h * G + G].to(F64)
                    err, tol = (got - o).abs(), 2.0 ** -8 * o.abs() + 2.0 ** -7 * w + 2.0 ** -16 * few
                    assert (err <= tol).all(), (b, h, float((err / tol).nan_to_num(math.inf).max()))
                    err2, w2 = err2 + float((err * err).sum()), w2 + float((w * w).sum())
                assert math.sqrt(err2 / w2) < most, (b, math.sqrt(err2 / w2))
            t0 += n


# bf16 rounds the output by 2^-9 of it on average at most; the weights' roundings are spread
# over many keys.  2^-8 is twice that.
NEAR = 2.0 ** -8

# nodes and heads that run each of the ways in which a call's rows are laid out: up to 32, up
# to 64 and more rows of a KV head, and sequences of both kinds (most of few rows)
LAYOUTS = {"few": ([5], 4, 1), "half": ([12], 8, 2), "full": ([64], 4, 2), "mixed": ([40, 2, 1, 3], 4, 1)}


@pytest.mark.parametrize("D,page", [(128, 64), (64, 16), (64, 8)])
@pytest.mark.parametrize("weight", [0.5, 0.8, 0.9])
@pytest.mark.parametrize("ctx", [4096, 16384, 33001])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_first_token_with_most_of_the_weight(layout, ctx, weight, D, page):
    nodes, Hq, Hkv = LAYOUTS[layout]
    call = Call(ctx + D, nodes, [ctx - 100 * b for b in range(len(nodes))], Hq, Hkv, D, page)
    for b in range(len(nodes)):
        call.dominant(b, weight)
    call.check(range(len(nodes)), NEAR)


@pytest.mark.parametrize("nodes,Hq,Hkv", [(5, 1, 1), (12, 4, 1), (32, 32, 8)])
def test_contexts_that_are_not_cut(nodes, Hq, Hkv):
    """As many items as the device has SMs: no context is cut over several of them."""
    B = -(-160 // Hkv)
    call = Call(nodes, [nodes] * B, [16384, 8200] + [9] * (B - 2), Hq, Hkv, 64, 32)
    for b in range(2):
        call.dominant(b, 0.9)
    call.check([0, 1, 2, B - 1], NEAR)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_equal_weights_behind_one_token(layout):
    """65536 tokens of the same score 11.2 nats below the first: half of the weight, none of
    it more than 2^-16 of the first's."""
    nodes, Hq, Hkv = LAYOUTS[layout]
    call = Call(1, nodes, [65536] * len(nodes), Hq, Hkv, 64, 64, spread=0.0)
    # (the first token's V takes away what the others add: the output is a small part of the
    # sum p |V| = 1 that the roundings are relative to)
    call.v[:] = 1.0
    for b in range(len(nodes)):
        call.score(b, 0, 1, 11.2)
        call.v[call.first[b]] = -1.0
    call.check(range(len(nodes)), NEAR)


@pytest.mark.parametrize("page", [32, 16, 8])
@pytest.mark.parametrize("power", [4, 8, 12, 16])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_values_of_another_scale_without_weight(layout, power, page):
    """32 tokens with next to no weight whose V is 2^4 to 2^16 times the others'."""
    nodes, Hq, Hkv = LAYOUTS[layout]
    call = Call(power, nodes, [4096 - 64 * b for b in range(len(nodes))], Hq, Hkv, 64, page)
    for b in range(len(nodes)):
        at = 640 + 32 * b
        call.score(b, at, at + 32, -40.0)
        call.v[call.first[b] + at:call.first[b] + at + 32] *= 2.0 ** power
    call.check(range(len(nodes)), NEAR)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_weight_that_moves_along_the_context(layout, D):
    """Scores that grow by 60 nats over the context, and that fall by as much: the reference
    of the weights has to follow, or the earlier tokens stay the ones that count."""
    nodes, Hq, Hkv = LAYOUTS[layout]
    for sign in (1, -1):
        call = Call(D, nodes, [3000] * len(nodes), Hq, Hkv, D, 16, spread=0.3)
        for b in range(len(nodes)):
            up = torch.linspace(-30, 30, 3000, device="cuda") * sign * math.sqrt(D) / 8.0
            call.k[call.first[b]:call.first[b] + 3000, :, 0] = up[:, None]
        call.check(range(len(nodes)), NEAR)


@pytest.mark.parametrize("power", [6, 9, 12])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_queries_with_one_large_component(layout, D, power):
    """A component of q that is 2^6 to 2^12 times the others, where K is 0: the others give the
    scores, and keep the bits that they have."""
    nodes, Hq, Hkv = LAYOUTS[layout]
    call = Call(power + D, nodes, [700] * len(nodes), Hq, Hkv, D, 16, spread=64.0)
    call.q[..., 1:] /= 16.0                              # scores N(0, 4)
    call.q[..., 0] = 2.0 ** (power - 4)
    call.check(range(len(nodes)), NEAR)


@pytest.mark.parametrize("context,tree", [(0.0, 80), (0.0, 120), (2.0 ** -70, 0), (2.0 ** 80, 0), (2.0 ** 110, 110)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_values_of_context_and_tree_far_apart(layout, D, context, tree):
    """V of the context nothing or tiny beside the tree's, or the other way round, or both near
    the largest numbers."""
    nodes, Hq, Hkv = LAYOUTS[layout]
    call = Call(D, nodes, [300] * len(nodes), Hq, Hkv, D, 16)
    call.v *= context
    call.tree_v *= 2.0 ** tree
    call.check(range(len(nodes)), NEAR)


@pytest.mark.parametrize("D,page", [(128, 64), (64, 16)])
@pytest.mark.parametrize("at", [0, 1000, 4095])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_one_token_with_nearly_all_the_weight(layout, at, D, page):
    """A token with 0.97 to 0.999 of the weight: its weight is not rounded, so the output's error
    is that of the other weights.  They are rounded by 2^-8 of at most 0.03, and those of its 31
    neighbours, which may be lost (below 2^-16 of it), make up 31 / 4096 of that 0.03 on
    average.  An error of e changes the rounding to bf16, whose steps are at least 2^-8 of a
    value, in a share of at most 2^8 e of the places: 2^8 (2^-8 + 31 / 4096) 0.03 = 0.09.  (A
    rounding of the token's own weight by 2^-9 would show in up to half of them.)"""
    nodes, Hq, Hkv = LAYOUTS[layout]
    call = Call(at + D, nodes, [4096] * len(nodes), Hq, Hkv, D, page)
    for b in range(len(nodes)):
        call.k[call.first[b] + at, :, 1:] = 0
        call.score(b, at, at + 1, math.log(99.0 * 4096) + 0.5)
    out, k, v, _ = call.run()
    G, t0, off, n_all = Hq // Hkv, 0, 0, 0
    for b, n in enumerate(nodes):
        rows = slice(call.first[b], call.first[b] + 4096)
        for h in range(Hkv):
            q = call.q16[t0:t0 + n, h * G:h * G + G].to(F64)
            kk = torch.cat([k[rows, h], call.tk16[t0:t0 + n, h].to(F64)])
            vv = torch.cat([v[rows, h], call.tv16[t0:t0 + n, h].to(F64)])
            x = torch.einsum("ngd,kd->ngk", q, kk) / math.sqrt(D)
            see = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
            x[:, :, 4096:] = x[:, :, 4096:].masked_fill(~see[:, None], -math.inf)
            p = x.softmax(-1)
            some = (p[..., at] > 0.97) & (p[..., at] < 0.999)      # (the cache rounds the key)
            assert some.float().mean() > 0.5
            differ = out[t0:t0 + n, h * G:h * G + G] != (p @ vv).to(B16)
            off, n_all = off + int(differ[some].sum()), n_all + int(some.sum()) * D
        t0 += n
    assert off <= 0.09 * n_all, (off, n_all)
