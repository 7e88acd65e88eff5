"""The serving operators together, as a decoder block uses them: projections of packed prompts, the
4-bit cache, attention over it, the output projection on top of the residual, and experts; then
decode steps, captured and replayed. Each result is compared with the float64 form of its own inputs
(the results before it), with the tolerances of the operators' own tests.
"""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_util import DEV, note, rel_frob
from paper_2607_07964_amd import kronq as K
from test_gpu_cache import TOL as TOL_ATTENTION
from test_gpu_served import BF16, BOTH, TOL, Layer, f64, rows_of

pytestmark = pytest.mark.gpu
D, HEADS, KV, DIM, PAGE, HIDDEN, EXPERTS, SEQS = 512, 8, 2, 128, 16, 448, 3, 3


class Block:
    def __init__(self):
        self.q = Layer(HEADS * DIM, D, 4, 128, BOTH, seed=1)
        self.k = Layer(KV * DIM, D, 4, 128, BOTH, seed=2)
        self.v = Layer(KV * DIM, D, 3, 128, BOTH, seed=3)
        self.o = Layer(D, HEADS * DIM, 4, 128, BOTH, seed=4, bias=False)
        self.up = Layer(HIDDEN, D, 2, 128, BOTH, seed=5, experts=EXPERTS)
        self.down = Layer(D, 896, 4, 128, BOTH, seed=6, experts=EXPERTS, bias=False)

    def step(self, s, hats=None):
        """One pass over the rows of s["x"]; every intermediate result."""
        lin = lambda la, x, **kw: K.kronq_online_linear(  # noqa: E731
            *la.one(), x, bias=None if la.bias_d is None else la.bias_d[0], **kw)
        x = s["x"]
        n = x.shape[0]
        r = {"q": lin(self.q, x), "k": lin(self.k, x), "v": lin(self.v, x)}
        k_hat, v_hat = hats or (None, None)
        K.kronq_cache_append(r["k"].view(n, KV, DIM), r["v"].view(n, KV, DIM), s["slots"], s["codes"],
                             s["params"], k_hat=k_hat, v_hat=v_hat)
        r["a"] = K.kronq_cache_attention(r["q"].view(n, HEADS, DIM), s["codes"], s["params"],
                                         s["table"], s["lengths"], starts=s.get("starts"),
                                         max_new=s.get("most")).view(n, -1)
        r["y"] = lin(self.o, r["a"], residual=x)
        # rows by expert (s["expert"]), and back
        order = torch.argsort(s["expert"], stable=True)
        offsets = (s["expert"][:, None] < torch.arange(EXPERTS + 1, device=DEV)).sum(0).to(torch.int32)
        r["offsets"], r["rows"] = offsets, r["y"].index_select(0, order)
        r["h"] = K.kronq_online_grouped(*self.up.args, *self.up.factors, r["rows"], offsets,
                                        bias=self.up.bias_d, act="silu", flags=BOTH)
        r["hh"] = torch.cat([r["h"], r["h"].flip(1)], 1)
        r["z"] = K.kronq_online_grouped(*self.down.args, *self.down.factors, r["hh"], offsets,
                                        residual=r["rows"], flags=BOTH)
        r["out"] = torch.empty_like(r["z"]).index_copy_(0, order, r["z"])
        return r

    def check(self, s, r, held, news):
        """held: the float64 keys and values of every sequence; news: its new tokens."""
        x = f64(s["x"])
        for name, la, arg, res in (("q", self.q, x, None), ("k", self.k, x, None),
                                   ("v", self.v, x, None), ("y", self.o, f64(r["a"]), x)):
            assert rel_frob(f64(r[name]), la.ref(arg, residual=res)) < TOL[BF16], name
        want, at = np.zeros((x.shape[0], HEADS, DIM)), 0
        q = f64(r["q"]).reshape(-1, HEADS, DIM)
        for (k, v), n in zip(held, news):
            want[at:at + n] = O.causal_attention(q[at:at + n], k, v, DIM ** -0.5)
            at += n
        assert rel_frob(f64(r["a"]), want.reshape(x.shape[0], -1)) < TOL_ATTENTION
        off = r["offsets"].tolist()
        rows, hh = f64(r["rows"]), f64(r["hh"])
        for name, la, arg, act, res in (("h", self.up, rows, "silu", None),
                                        ("z", self.down, hh, "none", rows)):
            for e in range(EXPERTS):
                cut = slice(off[e], off[e + 1])
                if off[e + 1] > off[e]:
                    ref = la.ref(arg[cut], act, None if res is None else res[cut], e)
                    assert rel_frob(f64(r[name])[cut], ref) < TOL[BF16], (name, e)


def start(prompts, room):
    """A cache whose pages lie in no order, with room for more tokens."""
    r = np.random.default_rng(5)
    need = [-(-(n + room) // PAGE) for n in prompts]
    order = r.permutation(sum(need))
    table = np.full((len(prompts), max(need)), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n], at = order[at:at + n], at + n
    codes, params = K.kronq_cache_empty(sum(need), KV, DIM, PAGE, DEV)
    return {"codes": codes, "params": params, "table": torch.from_numpy(table).to(DEV)}, table


def slot(table, b, t):
    return int(table[b, t // PAGE]) * PAGE + t % PAGE


@pytest.mark.parametrize("prompts", [[37, 1, 16], [130, 75, 3]])
def test_block_prompts_then_captured_decoding(prompts):
    K.load()
    block, turn = Block(), O.hadamard(DIM) / np.sqrt(DIM)
    s, table = start(prompts, 5)
    total = sum(prompts)
    s["x"] = rows_of(total, D, BF16, seed=7).to(DEV)
    s["slots"] = torch.tensor([slot(table, b, t) for b, n in enumerate(prompts) for t in range(n)],
                              device=DEV)
    s["starts"] = torch.tensor(np.cumsum([0] + prompts), dtype=torch.int32, device=DEV)
    s["lengths"] = torch.tensor(prompts, dtype=torch.int32, device=DEV)
    s["most"] = max(prompts)
    s["expert"] = torch.arange(total, device=DEV) * 5 % 7 % EXPERTS
    hats = [torch.zeros(total, KV, DIM, device=DEV) for _ in range(2)]
    note(f"block prompts={prompts}")
    r = block.step(s, hats)
    torch.cuda.synchronize()
    begin = np.cumsum([0] + prompts)
    held = [[f64(h)[begin[b]:begin[b + 1]] @ turn for h in hats] for b in range(SEQS)]
    block.check(s, r, held, prompts)

    # decoding: one graph, replayed with new rows, places and lengths, beside eager steps on a copy
    g = {"codes": s["codes"], "params": s["params"], "table": s["table"],
         "x": torch.zeros(SEQS, D, dtype=BF16, device=DEV),
         "slots": torch.zeros(SEQS, dtype=torch.int64, device=DEV),
         "lengths": torch.zeros(SEQS, dtype=torch.int32, device=DEV),
         "expert": torch.tensor([2, 0, 2], device=DEV)}
    e = {**g, "codes": g["codes"].clone(), "params": g["params"].clone()}
    hats = [torch.zeros(SEQS, KV, DIM, device=DEV) for _ in range(2)]

    def feed(i):
        g["x"].copy_(rows_of(SEQS, D, BF16, seed=50 + i))
        g["slots"].copy_(torch.tensor([slot(table, b, n + i) for b, n in enumerate(prompts)]))
        g["lengths"].copy_(torch.tensor([n + i + 1 for n in prompts], dtype=torch.int32))

    feed(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block.step(g, hats)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    note("block captured")
    with torch.cuda.graph(graph):
        captured = block.step(g, hats)
    for i in range(5):
        feed(i)
        graph.replay()
        torch.cuda.synchronize()
        eager = block.step(e)
        torch.cuda.synchronize()
        for name in captured:
            assert torch.equal(captured[name], eager[name]), (i, name)
        assert torch.equal(g["codes"], e["codes"]) and torch.equal(g["params"], e["params"])
        for b in range(SEQS):
            held[b] = [np.concatenate([t, f64(h)[b:b + 1] @ turn]) for t, h in zip(held[b], hats)]
        block.check(g, captured, held, [1] * SEQS)


def test_two_graphs_share_a_workspace():
    """Two captured calls with one workspace, replayed in turn on one stream."""
    K.load()
    la, lb = Layer(256, 512, 4, 128, BOTH, seed=8), Layer(512, 256, 3, 128, BOTH, seed=9)
    xa, xb = rows_of(40, 512, BF16, seed=1).to(DEV), rows_of(90, 256, BF16, seed=2).to(DEV)
    size = max(K.kronq_workspace_bytes(K.OP_LINEAR, 256, 512, 40),
               K.kronq_workspace_bytes(K.OP_LINEAR, 512, 256, 90))
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    ya = torch.zeros(40, 256, dtype=BF16, device=DEV)
    yb = torch.zeros(90, 512, dtype=BF16, device=DEV)
    calls = [lambda: K.kronq_online_linear(*la.one(), xa, y=ya, ws=ws),
             lambda: K.kronq_online_linear(*lb.one(), xb, y=yb, ws=ws)]
    note("two graphs, one workspace")
    graphs = []
    for call in calls:
        call()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call()
    want = ya.clone(), yb.clone()
    for i in range(3):
        ya.zero_(), yb.zero_()
        for k in ((0, 1), (1, 0), (0, 1, 0))[i]:
            graphs[k].replay()
        torch.cuda.synchronize()
        assert torch.equal(ya, want[0]) and torch.equal(yb, want[1])


@pytest.mark.parametrize("dim", [64, 128])
def test_prompts_into_rows_of_any_alignment(dim):
    """Outputs that begin on an odd element are stored one by one, and are the same."""
    n, heads = 150, 4
    q = torch.randn(n, heads, dim, generator=torch.Generator().manual_seed(3)).to(BF16).to(DEV)
    codes, params = K.kronq_cache_empty(10, 1, dim, 16, DEV)
    kv = torch.randn(2, n, 1, dim, generator=torch.Generator().manual_seed(4)).to(BF16).to(DEV)
    K.kronq_cache_append(kv[0], kv[1], torch.arange(n, device=DEV), codes, params)
    args = (codes, params, torch.arange(10, dtype=torch.int32, device=DEV)[None],
            torch.tensor([n], dtype=torch.int32, device=DEV))
    starts = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    note(f"prompts into odd rows dim={dim}")
    want = K.kronq_cache_attention(q, *args, starts=starts)
    odd = torch.full((n * (heads * dim + 3) + 1,), 3.0, dtype=BF16, device=DEV)
    rows = odd[1:].view(n, heads * dim + 3)
    K.kronq_cache_attention(q, *args, starts=starts,
                            out=rows[:, :heads * dim].unflatten(1, (heads, dim)))
    torch.cuda.synchronize()
    assert torch.equal(rows[:, :heads * dim], want.view(n, -1)) and bool(want.any())
    assert bool((rows[:, heads * dim:] == 3).all()) and float(odd[0]) == 3


@pytest.mark.parametrize("rotate,dim", [(True, 128), (True, 64), (False, 128)])
def test_append_rows_next_to_the_borders_of_the_grid(rotate, dim):
    """Rows of few small whole numbers, whose values fall on halves between two codes and whose
    scales are bf16 numbers exactly, beside rows of many sizes: the codes of fp64."""
    r = np.random.default_rng(dim)
    n = 1500
    rows = np.concatenate([r.integers(-7, 8, (n, dim)) * 2.0 ** r.integers(-3, 3, (n, 1)),
                           r.standard_normal((n, dim)) * np.exp(3 * r.standard_normal((n, 1))),
                           r.standard_normal((n, dim)) * np.exp(6 * r.standard_normal((n, dim)))])
    k = torch.from_numpy(rows).to(BF16).view(3 * n, 1, dim)
    codes, params = K.kronq_cache_empty(-(-3 * n // 64), 1, dim, 64, DEV)
    hats = [torch.zeros(3 * n, 1, dim, device=DEV) for _ in range(2)]
    note(f"append next to borders rotate={rotate} dim={dim}")
    K.kronq_cache_append(k.to(DEV), (-k).to(DEV), torch.arange(3 * n, device=DEV), codes, params,
                         rotate=rotate, k_hat=hats[0], v_hat=hats[1])
    torch.cuda.synchronize()
    for hat, t in zip(hats, (k, -k)):
        q, scale, zero, held = O.cache_grid(f64(t), rotate)
        assert np.array_equal(f64(hat), held.astype(np.float32).astype(np.float64))


@pytest.mark.parametrize("rows,first,last", [(260, 10, 200), (700, 33, 700), (9, 0, 9)])
def test_one_expert_of_some_rows(rows, first, last):
    """A single expert that begins inside a unit of 32 rows; the other rows keep what they hold."""
    la = Layer(256, 512, 4, 128, BOTH, seed=12)
    x = rows_of(rows, 512, BF16, seed=13)
    y = torch.full((rows, 256), 7.0, dtype=BF16, device=DEV)
    offsets = torch.tensor([first, last], dtype=torch.int32, device=DEV)
    note(f"one expert rows={rows} [{first}, {last})")
    K.kronq_online_grouped(*la.args, *la.factors, x.to(DEV), offsets, y, bias=la.bias_d, flags=BOTH)
    torch.cuda.synchronize()
    assert rel_frob(f64(y)[first:last], la.ref(f64(x)[first:last])) < TOL[BF16]
    assert bool((y[:first] == 7).all()) and bool((y[last:] == 7).all())


@pytest.mark.parametrize("d_out,rows", [(224, 5), (224, 33), (28672, 32), (28672, 33), (896, 6)])
@pytest.mark.parametrize("ydt", [BF16, torch.float32])
def test_outputs_of_28_m_by_one_and_by_four_workgroups(d_out, rows, ydt):
    """Both ways of the output side, with every part of its epilogue."""
    la = Layer(d_out, 256, 4, 128, BOTH, seed=14)
    x, res = rows_of(rows, 256, BF16, seed=15), rows_of(rows, d_out, ydt, seed=16)
    note(f"28 m outputs d_out={d_out} rows={rows} {ydt}")
    y = K.kronq_online_linear(*la.one(), x.to(DEV), bias=la.bias_d[0], act="gelu",
                              residual=res.to(DEV), out_dtype=ydt)
    torch.cuda.synchronize()
    assert rel_frob(f64(y), la.ref(f64(x), "gelu", f64(res))) < TOL[ydt]


@pytest.mark.parametrize("bits", [2, 3, 4, 8])
@pytest.mark.parametrize("groups", [1, 2, 3, 5, 9])
@pytest.mark.parametrize("ydt", [BF16, torch.float32])
def test_few_rows_and_few_groups(bits, groups, ydt):
    """Rows of W of few groups, whose loads end in any place of the rings; wide strides of W."""
    la = Layer(300, 128 * groups, bits, 128, 0, seed=17)
    x = rows_of(20, 128 * groups, BF16, seed=18)
    wide = torch.full((300, la.packed.shape[1] + 4), -1, dtype=torch.int32, device=DEV)
    wide[:, :la.packed.shape[1]] = la.packed.view(torch.int32)
    note(f"few groups bits={bits} groups={groups} {ydt}")
    for packed in (la.packed, wide[:, :la.packed.shape[1]]):
        y = K.kronq_online_linear(packed, *la.one()[1:], x.to(DEV), bias=la.bias_d[0], flags=0,
                                  out_dtype=ydt)
        torch.cuda.synchronize()
        assert rel_frob(f64(y), la.ref(f64(x))) < TOL[ydt]


@pytest.mark.parametrize("heads,dim,new,pad", [(4, 128, [1, 1, 1], 40), (8, 64, [90, 0, 40], 3),
                                               (4, 128, [70], 0)])
def test_attention_fills_tokens_of_no_sequence(heads, dim, new, pad):
    """Zeros before the first and behind the last sequence where out is made by the call; with a given
    out they stay as they are; the others are the same."""
    n = sum(new) + 2 * pad
    codes, params = K.kronq_cache_empty(8 * len(new), 1, dim, 16, DEV)
    kv = torch.randn(2, 128 * len(new), 1, dim, generator=torch.Generator().manual_seed(5)).to(BF16)
    K.kronq_cache_append(kv[0].to(DEV), kv[1].to(DEV), torch.arange(128 * len(new), device=DEV), codes,
                         params)
    table = torch.arange(8 * len(new), dtype=torch.int32, device=DEV).view(len(new), 8)
    lengths = torch.full((len(new),), 100, dtype=torch.int32, device=DEV)
    starts = torch.tensor(np.cumsum([pad] + new), dtype=torch.int32, device=DEV)
    q = torch.randn(n, heads, dim, generator=torch.Generator().manual_seed(6)).to(BF16).to(DEV)
    note(f"attention fills new={new} pad={pad}")
    junk = torch.full((n, heads, dim), float("nan"), dtype=BF16, device=DEV)
    del junk  # (what the allocator hands out next is not zero)
    a = K.kronq_cache_attention(q, codes, params, table, lengths, starts=starts, max_new=max(new))
    given = torch.full((n, heads, dim), 3.0, dtype=BF16, device=DEV)
    K.kronq_cache_attention(q, codes, params, table, lengths, starts=starts, max_new=max(new), out=given)
    torch.cuda.synchronize()
    own = slice(pad, n - pad)
    assert torch.equal(a[own], given[own]) and bool(a[own].any())
    for cut in (slice(0, pad), slice(n - pad, n)):
        assert not bool(a[cut].any()) and bool((given[cut] == 3).all())
