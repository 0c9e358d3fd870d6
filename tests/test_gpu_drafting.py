"""Drafted trees as a server drives them: plan, products (8 or 4 bits), keys by slots, attention of the trees, accepted paths,
pages given back, the next step on what was kept; in a graph, on two streams, with ordinary steps between.

Against binary64 in two parts, so that a rounding before the second quantisation cannot move one of its codes.  The attended
values: x is quantised by the library and decoded exactly; a product of K terms in binary32 loses K 2^-23 of the terms' magnitudes and
half a step u = 2^-11 in the rounding to fp16, a rotation half a step more, so every score has a bound; the attended value is off by
exp(2 x the largest of them) - 1 and the rounding u of a probability, times the mean of |v|, by the mean of v's own bound, and by half
a step.  The outputs: the product on the attended values that the block had.
"""
import threading

import pytest
import torch

from paper_2311_01305_b200 import aweq, calibrate, serve, synth

from .test_gpu_mx4 import stands_for

pytestmark = pytest.mark.gpu

U, TINY, HEADS, D, PAGE = 2.0 ** -11, 2.0 ** -25, 12, 64, 16
FORMATS = [None, "e8m0", "e4m3"]


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module")
def layer():
    wl = synth.workloads(1.0 / 512)["opt125m_model_w8a8"]
    X, W = synth.generate(wl, "cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    bias = {n: 0.1 * torch.randn(W[n].shape[0], generator=g, device="cuda").to(W[n].dtype) for n in ("q", "v", "o")}
    cal = calibrate.LayerCalibrator(wl, 8, X, W, bias)
    cal.run()
    return cal, X["attn_in"], W, bias


def make_block(layer, fmt, pages, rope=None):
    cal, _, W, bias = layer
    return serve.AttentionBlock(cal, HEADS, pages, PAGE, rope, fmt=fmt, W=W if fmt else None, bias=bias if fmt else None)


def weights(block, cal, names):
    """The linears of a block as binary64 matrix and bias."""
    if block.fmt:
        lin = block.qkv if len(names) == 3 else block.o
        return stands_for(lin.weight), lin.bias.double()
    out = [cal.out[n] for n in names]
    return (torch.cat([(o["codes"].double() - o["zp"].double()[:, None]) * o["step"].double()[:, None] for o in out]),
            torch.cat([o["bias_f32"].double() for o in out]))


def decoded(block, x, rinv):
    """What the quantised x stands for, binary64."""
    x = x.contiguous()
    if block.fmt:
        return stands_for(aweq.MX4(*x.shape, block.fmt).quantise(x, rinv))
    codes, step, zp = torch.empty(x.shape, dtype=torch.uint8, device="cuda"), torch.empty(x.shape[0], device="cuda"), i32([0] * x.shape[0])
    aweq.aweq_quant_act(x, rinv, 8, aweq.PER_ROW, None, codes, step, zp)
    return (codes.double() - zp.double()[:, None]) * step.double()[:, None]


def product(x, w, b):
    """x w^T + b and its bound in binary32, rounded to fp16."""
    y, size = x @ w.t() + b, x.abs() @ w.abs().t() + b.abs()
    return y, (x.shape[1] + 4) * 2.0 ** -23 * size + U * y.abs() + TINY


def rotated(rope, y, e, pos):
    if rope is None:
        return y, e
    cs = rope.double()[pos][:, None]
    c, s = cs[..., :D // 2], cs[..., D // 2:]
    turn = lambda a, b, c, s: torch.cat([a * c - b * s, a * s + b * c], -1)  # noqa: E731
    z = turn(y[..., :D // 2], y[..., D // 2:], c, s)
    bound = turn(e[..., :D // 2], -e[..., D // 2:], c.abs(), s.abs())[..., :D // 2], turn(e[..., :D // 2], e[..., D // 2:], c.abs(), s.abs())[..., D // 2:]
    return z, torch.cat(bound, -1) + U * z.abs() + 2.0 ** -22 * (y.abs() + y.roll(D // 2, -1).abs()) + TINY


def attended(block, layer, z, pos, sees):
    """Attention of the last tokens of z [tokens, C], one for each row of ``sees`` [n, tokens], with its bound."""
    cal, n = layer[0], sees.shape[0]
    y, e = product(decoded(block, z, block.rinv["attn_in"]), *weights(block, cal, ("q", "k", "v")))
    (q, k, v), (eq, ek, ev) = ([t.unflatten(1, (HEADS, D)) for t in s.split(HEADS * D, 1)] for s in (y, e))
    q, eq = rotated(block.rope, q[-n:], eq[-n:], pos[-n:])
    k, ek = rotated(block.rope, k, ek, pos)
    mm = lambda a, b: torch.einsum("ihd,jhd->hij", a, b) * D ** -0.5  # noqa: E731
    score = mm(q, k).masked_fill(~sees, float("-inf"))
    off = mm(eq, k.abs()) + mm(q.abs() + eq, ek) + (D + 4) * 2.0 ** -23 * mm(q.abs(), k.abs())
    off = off.masked_fill(~sees, 0.0).amax(-1, keepdim=True)
    p = torch.softmax(score, -1)
    mean = lambda p, v: torch.einsum("hij,jhd->ihd", p, v)  # noqa: E731
    out = mean(p, v)
    # (2^-16: the exponentials and rescalings of a few hundred keys in binary32)
    tol = mean(p * (torch.expm1(2 * off) + U + 2.0 ** -16), v.abs() + ev) + mean(p, ev) + U * out.abs() + TINY
    return out, tol


class Recorded(aweq.TreeAttention):
    """Keeps what it answered."""

    def __call__(self, *args, **kw):
        out = super().__call__(*args, **kw)
        self.seen = out.clone()
        return out


class RecordedSteps(aweq.PrefixAttention):
    def __call__(self, *args, **kw):
        out = super().__call__(*args, **kw)
        self.seen = out.clone()
        return out


def check_output(block, layer, att, out):
    want, tol = product(decoded(block, att.flatten(1), block.rinv["o_in"]), *weights(block, layer[0], ("o",)))
    assert ((out.double() - want).abs() <= tol).all()


def tree(rng, n):
    """A tree of n nodes: every node's parent, depth, and itself with those above it; a path from a root."""
    up, depth, sees = [], [], torch.zeros(n, n, dtype=torch.bool)
    for i in range(n):
        up.append(int(torch.randint(max(-1, i - 6), i, (1,), generator=rng)) if i else -1)
        if up[i] >= 0:
            sees[i] = sees[up[i]]
        sees[i, i] = True
        depth.append(int(sees[i].sum()) - 1)
    path = sees[int(torch.randint(0, n, (1,), generator=rng))].nonzero().flatten().tolist() if n else []
    return up, depth, sees, path


def drawn(rng, tokens, n_seq, nodes, rows):
    """A step's drafts (ragged, one sequence without any), padded to ``rows``, and what the calls take."""
    trees = [tree(rng, int(torch.randint(0 if b == 1 else 1, 1 if b == 1 else nodes + 1, (1,), generator=rng))) for b in range(n_seq)]
    n = [len(t[0]) for t in trees]
    flat = sum((t[0] for t in trees), [])
    x = torch.full((rows, tokens.shape[1]), float("nan"), dtype=tokens.dtype, device="cuda")
    x[:len(flat)] = tokens[torch.randint(0, tokens.shape[0], (len(flat),), generator=rng).cuda()]
    return trees, dict(n=i32(n), parent=i32(flat + [-1] * (rows - len(flat))), path=i32([t[3] + [0] * (nodes - len(t[3])) for t in trees]),
                       n_path=i32([len(t[3]) for t in trees]), back=i32([len(t[3]) - m for t, m in zip(trees, n)]), x=x)


class Server:
    """A block, the pool of its pages, tables, plans and a prefix."""

    def __init__(self, block, layer, n_seq, nodes, rows, prefix, per_seq, pages, kind=aweq.TreeAttention):
        shared = -(-prefix // PAGE)
        order = pages[torch.randperm(pages.numel(), generator=torch.Generator().manual_seed(5)).cuda()]
        self.block, self.n_seq, self.nodes, self.rows, self.prefix = block, n_seq, nodes, rows, prefix
        self.prefix_pages = order[:shared].clone()
        ring = torch.zeros(block.cache.k.shape[0], dtype=torch.int32, device="cuda")
        ring[:order.numel() - shared] = order[shared:]
        self.pool = aweq.PagePool(ring.numel(), PAGE, ring=ring, state=torch.tensor([0, order.numel() - shared], device="cuda"))
        self.table = torch.full((n_seq, per_seq), -1, dtype=torch.int32, device="cuda")
        if prefix:
            block(layer[1][:prefix], block.attention(1, prefix, max_own=prefix), self.prefix_pages.view(1, -1), i32([prefix]),
                  torch.arange(prefix, dtype=torch.int32, device="cuda"), torch.zeros(prefix, dtype=torch.int32, device="cuda"))
        self.attend = kind(block.cache, self.prefix_pages, prefix, HEADS, n_seq, rows, nodes, per_seq * PAGE)
        self.grown, self.kept = aweq.StepPlan(n_seq, rows, nodes), aweq.StepPlan(n_seq, 0)
        self.kept.own_len.zero_()
        self.st = aweq.new_status()

    def step(self, n, parent, path, n_path, back, x):
        self.pool.plan(self.table, self.kept.own_len, n, self.grown, first=self.prefix, parent=parent, st=self.st)
        out = self.block.verify(x, self.attend, self.table, self.grown, self.st)
        aweq.aweq_kv_accept(self.block.cache, self.table, self.kept.own_len, path, n_path, self.st)
        self.pool.plan(self.table, self.grown.own_len, back, self.kept, st=self.st)
        return out

    def fine(self):
        return not self.st.any()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n_seq,nodes,prefix,with_rope", [(5, 20, 70, True), (3, 70, 0, False), (1, 1, 16, True)])
def test_drafted_steps_match_the_dequantised_layer(layer, fmt, n_seq, nodes, prefix, with_rope):
    rng = torch.Generator().manual_seed(11)
    tokens, steps, rows, per_seq = layer[1], 3, n_seq * nodes + 5, -(-4 * nodes // PAGE)
    rope = aweq.aweq_rope_table(D, 512) if with_rope else None
    n_pages = -(-prefix // PAGE) + n_seq * per_seq
    block = make_block(layer, fmt, n_pages + 2, rope)
    server = Server(block, layer, n_seq, nodes, rows, prefix, per_seq, torch.arange(n_pages, dtype=torch.int32, device="cuda"), Recorded)
    kept = [tokens[:prefix]] * n_seq
    for _ in range(steps):
        trees, call = drawn(rng, tokens, n_seq, nodes, rows)
        out = server.step(**call)
        at = 0
        for b, (up, depth, sees, path) in enumerate(trees):
            if not up:
                continue
            old, x = kept[b].shape[0], call["x"][at:at + len(up)]
            pos = torch.cat([torch.arange(old), old + torch.tensor(depth)]).cuda()
            want, tol = attended(block, layer, torch.cat([kept[b], x]), pos, torch.cat([torch.ones(len(up), old, dtype=torch.bool), sees], 1).cuda())
            got = server.attend.seen[at:at + len(up)]
            assert ((got.double() - want).abs() <= tol).all()
            check_output(block, layer, got, out[at:at + len(up)])
            kept[b] = torch.cat([kept[b], x[torch.tensor(path, device="cuda")]])
            at += len(up)
        assert server.kept.own_len.tolist() == [k.shape[0] - prefix for k in kept]
    # an ordinary token of each sequence on what the trees left
    plan, x = aweq.StepPlan(n_seq, n_seq), tokens[prefix:prefix + n_seq].contiguous()
    server.pool.plan(server.table, server.kept.own_len, i32([1] * n_seq), plan, first=prefix, st=server.st)
    attend = RecordedSteps(block.cache, server.prefix_pages, prefix, HEADS, n_seq, 1, per_seq * PAGE)
    out = block(x, attend, server.table, plan.own_len, plan.pos, plan.seq, server.st)
    for b in range(n_seq):
        z = torch.cat([kept[b], x[b:b + 1]])
        want, tol = attended(block, layer, z, torch.arange(z.shape[0], device="cuda"), torch.ones(1, z.shape[0], dtype=torch.bool, device="cuda"))
        assert ((attend.seen[b:b + 1].double() - want).abs() <= tol).all()
    check_output(block, layer, attend.seen, out)
    assert server.fine()
    # pages that nobody had: as they were made
    assert not block.cache.k[n_pages:].any() and not block.cache.v[n_pages:].any()


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_captured_step_answers_as_the_calls_do(layer, fmt):
    n_seq, nodes, rows, prefix, per_seq = 4, 12, 60, 33, 4
    n_pages = 3 + n_seq * per_seq
    rope = aweq.aweq_rope_table(D, 256)
    pages = torch.arange(n_pages, dtype=torch.int32, device="cuda")
    servers = [Server(make_block(layer, fmt, n_pages, rope), layer, n_seq, nodes, rows, prefix, per_seq, pages) for _ in range(2)]
    rng = torch.Generator().manual_seed(2)
    drafts = [drawn(rng, layer[1], n_seq, nodes, rows) for _ in range(4)]
    # the first step by calls on both, the others as a graph on one of them
    static = {k: v.clone() for k, v in drafts[0][1].items()}
    for s in servers:
        s.step(**static)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        replayed = servers[1].step(**static)
    for trees, call in drafts[1:]:
        for k, v in call.items():
            static[k].copy_(v)
        graph.replay()
        out, n = servers[0].step(**call), sum(len(t[0]) for t in trees)
        assert torch.equal(out[:n], replayed[:n])
        assert torch.equal(servers[0].kept.own_len, servers[1].kept.own_len) and torch.equal(servers[0].table, servers[1].table)
    assert torch.equal(servers[0].block.cache.k, servers[1].block.cache.k) and all(s.fine() for s in servers)


def test_two_streams_draft_at_a_time(layer):
    """One block, each stream with pages, plans and an attention of its own, against the same steps alone."""
    n_seq, nodes, rows, prefix, per_seq = 6, 24, 144, 50, 6
    n_pages = 4 + n_seq * per_seq
    rng = torch.Generator().manual_seed(4)
    drafts = [[drawn(rng, layer[1], n_seq, nodes, rows) for _ in range(3)] for _ in range(2)]
    rope = aweq.aweq_rope_table(D, 512)
    block = make_block(layer, "e8m0", 2 * n_pages, rope)
    run = lambda server, steps: [server.step(**call)[:sum(len(t[0]) for t in trees)].clone() for trees, call in steps]  # noqa: E731
    made = lambda i: Server(block, layer, n_seq, nodes, rows, prefix, per_seq, torch.arange(i * n_pages, (i + 1) * n_pages, dtype=torch.int32, device="cuda"))  # noqa: E731
    alone = [run(made(i), drafts[i]) for i in range(2)]
    torch.cuda.synchronize()
    servers, got = [made(i) for i in range(2)], [None, None]
    torch.cuda.synchronize()

    def serve_one(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            got[i] = run(servers[i], drafts[i])
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=serve_one, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert all(torch.equal(a, b) for one, two in zip(alone, got) for a, b in zip(one, two)) and all(s.fine() for s in servers)


def test_a_block_in_4_bits_keeps_what_it_was_made_of(layer):
    cal, tokens, W, bias = layer
    own = {n: w.clone() for n, w in W.items()}
    block = serve.AttentionBlock(cal, HEADS, 4, PAGE, fmt="e4m3", W=own, bias=bias)
    table = i32([[0, 1], [2, 3]])
    call = lambda: block(tokens[:6].contiguous(), block.attention(2, 3, max_own=32), table, i32([3, 3]), i32([0, 1, 2] * 2), i32([0] * 3 + [1] * 3))  # noqa: E731
    want = call()
    for w in own.values():
        w.zero_()
    assert torch.equal(call(), want)


def test_the_rounding_of_the_weights_has_mean_zero_on_the_calibration_inputs(layer):
    """Eq. 15: with the corrected bias the mean output on the calibration's tokens is the 16-bit layer's, but for binary32 sums:
    K 2^-23 of the magnitudes for the sum of the rounding, for E[x/s], and for the bias."""
    cal, tokens, W, bias = layer
    lin = serve.joint_linear_mx4(cal, ("q", "k", "v"), W, "e8m0", bias)
    w = torch.cat([W[n] for n in ("q", "k", "v")]).double()
    b = torch.cat([bias["q"].double(), torch.zeros(W["k"].shape[0], device="cuda").double(), bias["v"].double()])
    o = cal.out["attn_in"]
    mu = o["mu_hat"].double()
    got = stands_for(lin.weight) @ mu + lin.bias.double()
    want = (w * o["s"].double()) @ mu + b
    size = (w * o["s"].double()).abs() @ mu.abs() + (stands_for(lin.weight)).abs() @ mu.abs() + b.abs()
    assert ((got - want).abs() <= (w.shape[1] + 4) * 2.0 ** -23 * size).all()


@pytest.mark.parametrize("wrong", ["rows", "plan", "mask", "cache", "kind", "format", "weights"])
def test_refusals(layer, wrong):
    block = make_block(layer, "e8m0", 8)
    x = torch.zeros((8, block.qkv.C_in), dtype=block.dtype, device="cuda")
    plan, attend = aweq.StepPlan(2, 8, 4), block.drafts(2, 8, 4, max_own=64)
    table = i32([[0, 1], [2, 3]])
    with pytest.raises(ValueError):
        if wrong == "rows":
            block.verify(x[:7], attend, table, plan)
        elif wrong == "plan":
            block.verify(x, attend, table, aweq.StepPlan(3, 8, 4))
        elif wrong == "mask":
            block.verify(x, attend, table, aweq.StepPlan(2, 8))
        elif wrong == "cache":
            block.verify(x, make_block(layer, "e8m0", 8).drafts(2, 8, 4, max_own=64), table, plan)
        elif wrong == "kind":
            block.verify(x, block.attention(2, 4), table, plan)
        elif wrong == "format":
            make_block(layer, "e5m2", 8)
        else:
            serve.AttentionBlock(layer[0], HEADS, 8, fmt="e8m0")
    assert not block.cache.k.any()


def test_the_example_runs(capsys):
    assert 0.0 < serve.drafting(n_seq=4, prefix=100, steps=3, nodes=6)
    assert "4 sequences, trees of up to 6 drafted tokens, 3 steps" in capsys.readouterr().out
