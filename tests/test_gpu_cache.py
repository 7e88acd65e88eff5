"""The 4-bit key/value cache (kronq_cache_append) and the attention over it
(kronq_cache_attention) through the C ABI against the float64 oracle.

Codes, scales and zeros are compared exactly: the grid is defined in fp64. Attention: the result is
rounded to bf16 (at most 2^-8 of each value); a weight p s_t is rounded to fp16 (2^-11, independent
from token to token) and its score is off by the rounding of q, 2^-11 of the sum of |q_d k_d| times
the scale in the worst case and its square root over dim in the mean, which for the scores of these
tests (|q|, |k| of about sqrt(dim), scale 1 / sqrt(dim)) stays below 2^-11 * 4, taken for every
weight: 2^-8 + 2^-11 + 4 * 2^-11, relative Frobenius.
"""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_util import DEV, note, rel_frob
from paper_2607_07964_amd import kronq as K

pytestmark = pytest.mark.gpu
TOL = 2.0 ** -8 + 5 * 2.0 ** -11
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    K.load()
    assert torch.cuda.is_available(), "GPU tests need an MI355X"


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def randn(*size, seed=0, dtype=BF16):
    return torch.randn(*size, generator=torch.Generator().manual_seed(seed)).to(dtype)


def words(t):
    return t.cpu().numpy().view(np.uint32)


# ------------------------------------------------------------------------------------------ append
def grid_check(k, v, slots, codes, params, before, hats, page, rotate):
    """The cache after an append against the oracle, word for word, and its untouched places."""
    c, p = words(codes), words(params)
    c0, p0 = (words(t) for t in before)
    pages, kv = p.shape[:2]
    dim = k.shape[-1]
    want_c, want_p = c0.copy(), p0.copy()
    for part, (t, hat) in enumerate(zip((k, v), hats)):
        q, scale, zero, held = O.cache_grid(f64(t), rotate)
        for i, slot in enumerate(slots):
            if slot < 0 or slot >= pages * page:
                continue
            pg, off = divmod(int(slot), page)
            for h in range(kv):
                whole = np.zeros((page, dim), dtype=np.int64)
                whole[off] = q[i, h]
                mine = np.zeros((page, dim), dtype=np.int64)
                mine[off] = 15
                mask = O.cache_words(mine, part)
                want_c[pg, h, part] = (want_c[pg, h, part] & ~mask) | O.cache_words(whole, part)
                bits = np.float32(scale[i, h]).view(np.uint32)
                want_p[pg, h, part, off] = bits | np.uint32(zero[i, h])
            if hat is not None:
                assert np.array_equal(f64(hat[i]), held[i].astype(np.float32).astype(np.float64))
    assert np.array_equal(p, want_p)
    assert np.array_equal(c, want_c)


@pytest.mark.parametrize("dim,kv,page,tokens,rotate,dtype", [
    (128, 2, 16, 1, True, BF16), (128, 8, 64, 37, True, BF16), (128, 1, 32, 60, False, BF16),
    (64, 3, 16, 33, True, FP32), (64, 2, 128, 5, False, FP32), (128, 2, 256, 100, True, FP32),
])
def test_append_matches_the_grid(dim, kv, page, tokens, rotate, dtype):
    pages = -(-tokens // page) + 2
    codes, params = K.kronq_cache_empty(pages, kv, dim, page, DEV)
    codes.random_(-2 ** 31, 2 ** 31 - 1)
    params.random_(-2 ** 31, 2 ** 31 - 1)
    before = codes.clone(), params.clone()
    k, v = randn(tokens, kv, dim, seed=1, dtype=dtype), randn(tokens, kv, dim, seed=2, dtype=dtype)
    k[..., 3] *= 20
    slots = np.random.default_rng(tokens).permutation(pages * page)[:tokens]
    hats = [torch.full((tokens, kv, dim), float("nan"), device=DEV) for _ in range(2)]
    note(f"append dim={dim} kv={kv} page={page} tokens={tokens} rotate={rotate} {dtype}")
    K.kronq_cache_append(k.to(DEV), v.to(DEV), torch.from_numpy(slots).to(DEV), codes, params,
                         rotate=rotate, k_hat=hats[0], v_hat=hats[1])
    torch.cuda.synchronize()
    grid_check(k, v, slots, codes, params, before, hats, page, rotate)


def test_append_leaves_out_slots_that_do_not_exist():
    codes, params = K.kronq_cache_empty(3, 2, 128, 16, DEV)
    codes.fill_(0x12345678), params.fill_(7)
    before = codes.clone(), params.clone()
    slots = np.array([-1, 5, 48, 47, -2 ** 40, 2 ** 40, 0])
    k, v = randn(7, 2, 128, seed=3), randn(7, 2, 128, seed=4)
    hats = [torch.full((7, 2, 128), 5.0, device=DEV) for _ in range(2)]
    note("append with slots outside the cache")
    K.kronq_cache_append(k.to(DEV), v.to(DEV), torch.from_numpy(slots).to(DEV), codes, params,
                         k_hat=hats[0], v_hat=hats[1])
    torch.cuda.synchronize()
    grid_check(k, v, slots, codes, params, before, (None, None), 16, True)
    for i in (0, 2, 4, 5):
        assert bool((hats[0][i] == 5).all()) and bool((hats[1][i] == 5).all())


def test_append_special_rows():
    """Zeros, one-sided rows, borders between codes, tiny and huge values, NaN and infinity."""
    dim = 64
    rows = np.zeros((9, dim), dtype=np.float32)
    rows[1] = np.linspace(1, 2, dim)              # all positive: zero code 0
    rows[2] = -np.linspace(1, 2, dim)             # all negative: zero code 15
    rows[3] = (np.arange(dim) % 31 - 15) * 0.5    # scale 1: halves lie between two codes
    rows[4] = np.linspace(-1, 1, dim) * 1e-35     # below the smallest scale
    rows[5] = np.linspace(-1, 1, dim) * 1e30
    rows[6] = rows[7] = rows[8] = np.linspace(-1, 1, dim)
    rows[7, 3], rows[8, 60] = np.nan, np.inf
    k = torch.from_numpy(rows).view(9, 1, dim)
    for rotate in (False, True):
        codes, params = K.kronq_cache_empty(1, 1, dim, 16, DEV)
        before = codes.clone(), params.clone()
        hats = [torch.zeros(9, 1, dim, device=DEV) for _ in range(2)]
        slots = np.arange(9)
        note(f"append special rows rotate={rotate}")
        K.kronq_cache_append(k.to(DEV), k.flip(0).to(DEV), torch.from_numpy(slots).to(DEV), codes,
                             params, rotate=rotate, k_hat=hats[0], v_hat=hats[1])
        torch.cuda.synchronize()
        assert torch.isnan(hats[0][7:]).all() and torch.isnan(hats[1][:2]).all()
        fine = K.kronq_cache_empty(1, 1, dim, 16, DEV)
        K.kronq_cache_append(k[:7].to(DEV), k[:7].to(DEV), torch.arange(7, device=DEV), *fine,
                             rotate=rotate)
        torch.cuda.synchronize()
        grid_check(k[:7], k[:7], slots[:7], *fine, before, (hats[0][:7], None), 16, rotate)


def test_append_strided_tokens():
    """k and v as slices of one fused projection."""
    qkv = randn(21, 3 * 2 * 128, seed=9).to(DEV)
    k = qkv[:, 256:512].unflatten(1, (2, 128))
    v = qkv[:, 512:].unflatten(1, (2, 128))
    codes, params = K.kronq_cache_empty(2, 2, 128, 16, DEV)
    before = codes.clone(), params.clone()
    slots = np.arange(31, 10, -1)
    note("append of strided tokens")
    K.kronq_cache_append(k, v, torch.from_numpy(slots.copy()).to(DEV), codes, params)
    torch.cuda.synchronize()
    grid_check(k, v, slots, codes, params, before, (None, None), 16, True)


# --------------------------------------------------------------------------------------- attention
class Cache:
    """Sequences of the given lengths appended to a cache with shuffled pages."""

    def __init__(self, lengths, kv, dim, page, rotate, seed=0, spare=2, wide=0):
        r = np.random.default_rng(seed)
        self.lengths, self.kv, self.dim, self.page, self.rotate = lengths, kv, dim, page, rotate
        need = [-(-n // page) for n in lengths]
        pages = sum(need) + spare
        order = r.permutation(pages)
        cols = max(max(need), 1) + wide
        self.table = np.full((len(lengths), cols), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        total = sum(lengths)
        self.k = randn(total, kv, dim, seed=seed + 1)
        self.v = randn(total, kv, dim, seed=seed + 2) + 0.25
        self.codes, self.params = K.kronq_cache_empty(pages, kv, dim, page, DEV)
        self.codes.random_(-2 ** 31, 2 ** 31 - 1)  # what nobody wrote may be anything
        self.params.fill_(0x7FC07FC0)              # (NaN scales)
        slots = [int(self.table[b, t // page]) * page + t % page
                 for b, n in enumerate(lengths) for t in range(n)]
        if total:
            K.kronq_cache_append(self.k.to(DEV), self.v.to(DEV),
                                 torch.tensor(slots, dtype=torch.int64, device=DEV), self.codes,
                                 self.params, rotate=rotate)
        self.begin = np.cumsum([0] + list(lengths))
        h = O.hadamard(dim) / np.sqrt(dim) if rotate else np.eye(dim)
        self.held = [O.cache_grid(f64(t), rotate)[3] @ h if total else None
                     for t in (self.k, self.v)]

    def dev(self):
        return (self.codes, self.params, torch.from_numpy(self.table).to(DEV),
                torch.tensor(self.lengths, dtype=torch.int32, device=DEV))

    def ref(self, q, starts, scale=None):
        out = np.zeros(q.shape)
        for b, n in enumerate(self.lengths):
            a, e = starts[b], starts[b + 1]
            k, v = (t[self.begin[b]:self.begin[b + 1]] if n else np.zeros((0, self.kv, self.dim))
                    for t in self.held)
            out[a:e] = O.causal_attention(q[a:e], k, v, scale or self.dim ** -0.5)
        return out


@pytest.mark.parametrize("lengths,heads,kv,dim,page,rotate", [
    ([1], 4, 4, 128, 16, True), ([1, 2, 31], 8, 2, 128, 16, True),
    ([32, 33, 64, 65], 8, 8, 64, 32, False), ([127, 128, 129, 300], 28, 4, 128, 64, True),
    ([1000, 3, 517], 32, 8, 128, 64, True), ([700], 8, 1, 64, 128, True),
    ([2500], 17, 1, 128, 16, True), ([40, 900], 48, 1, 64, 64, False),
    ([257] * 5, 6, 6, 128, 256, False),
])
def test_decode_lengths_and_heads(lengths, heads, kv, dim, page, rotate):
    c = Cache(lengths, kv, dim, page, rotate)
    q = randn(len(lengths), heads, dim, seed=7)
    note(f"decode {lengths} heads={heads}/{kv} dim={dim} page={page}")
    o = K.kronq_cache_attention(q.to(DEV), *c.dev(), rotate=rotate)
    torch.cuda.synchronize()
    assert rel_frob(f64(o), c.ref(f64(q), np.arange(len(lengths) + 1))) < TOL


@pytest.mark.parametrize("lengths,new,heads,kv,dim,page", [
    ([5, 40, 1], [5, 40, 1], 4, 2, 128, 16),          # whole prompts
    ([70, 200], [33, 7], 8, 2, 64, 32),               # chunks after what is cached
    ([129, 64], [129, 63], 6, 6, 128, 64),
    ([300], [300], 7, 1, 128, 64),                    # rows of a head group over tile borders
    ([513, 20, 90], [100, 20, 1], 8, 1, 64, 16),
    ([0, 30, 0], [0, 30, 0], 4, 4, 128, 16),          # empty sequences
])
def test_prompts_are_causal(lengths, new, heads, kv, dim, page):
    c = Cache(lengths, kv, dim, page, True, seed=3)
    starts = np.cumsum([0] + new)
    q = randn(int(starts[-1]), heads, dim, seed=8)
    note(f"prompts {lengths} new={new} heads={heads}/{kv} dim={dim}")
    for most in (max(new), 1):  # a small max_new only sizes the launch
        o = K.kronq_cache_attention(q.to(DEV), *c.dev(),
                                    torch.tensor(starts, dtype=torch.int32, device=DEV),
                                    max_new=most)
        torch.cuda.synchronize()
        assert rel_frob(f64(o), c.ref(f64(q), starts)) < TOL


def test_queries_that_see_nothing_and_tokens_of_no_sequence():
    """More new tokens than cached ones: the first see nothing and give zeros. Rows of out outside
    every sequence stay as they were."""
    c = Cache([3, 0], 2, 64, 16, True, seed=5)
    starts = np.array([2, 8, 9])
    q = randn(11, 4, 64, seed=9)
    out = torch.full((11, 4, 64), 7.0, dtype=BF16, device=DEV)
    note("queries that see nothing")
    K.kronq_cache_attention(q.to(DEV), *c.dev(), torch.tensor(starts, dtype=torch.int32, device=DEV),
                            max_new=6, out=out)
    torch.cuda.synchronize()
    o = f64(out)
    assert np.all(o[[0, 1, 9, 10]] == 7.0)
    assert np.all(o[2:5] == 0.0) and np.all(o[8] == 0.0)
    assert rel_frob(o[5:8], c.ref(f64(q), starts)[5:8]) < TOL


def test_nan_behind_the_mask_and_in_sight():
    """A NaN value row is seen by the queries after it and by no earlier one, and by no other head."""
    c = Cache([100], 2, 128, 16, True, seed=6)
    slot = int(c.table[0, 60 // 16]) * 16 + 60 % 16
    c.params[slot // 16, 1, 1, slot % 16] = 0x7FC00000
    q = randn(100, 4, 128, seed=10)
    starts = np.array([0, 100])
    note("a NaN value row in a prompt")
    o = K.kronq_cache_attention(q.to(DEV), *c.dev(), torch.tensor(starts, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    ref, o = c.ref(f64(q), starts), f64(o)
    assert np.isnan(o[60:, 2:]).all()
    o[60:, 2:] = ref[60:, 2:]
    assert rel_frob(o, ref) < TOL


def test_pages_that_do_not_exist_are_not_seen():
    c = Cache([64, 40], 2, 64, 16, False, seed=11)
    q = randn(2, 2, 64, seed=12)
    codes, params, table, lengths = c.dev()
    for page in (-1, codes.shape[0], 2 ** 31 - 1):
        table[0, 1] = page
        note(f"a page outside the cache: {page}")
        o = K.kronq_cache_attention(q.to(DEV), codes, params, table, lengths, rotate=False)
        torch.cuda.synchronize()
        k, v = (np.concatenate((t[:16], t[32:64])) for t in c.held)
        ref = np.concatenate((O.causal_attention(f64(q)[:1], k, v, 0.125),
                              c.ref(f64(q), np.arange(3))[1:]))
        assert rel_frob(f64(o), ref) < TOL
    lengths[:] = torch.tensor([10 ** 9, -5], dtype=torch.int32)  # cut to the table, and to nothing
    note("lengths outside the table")
    o = K.kronq_cache_attention(q.to(DEV), codes, params, table, lengths, rotate=False)
    torch.cuda.synchronize()
    assert rel_frob(f64(o)[0], ref[0]) < TOL and np.all(f64(o)[1] == 0.0)


@pytest.mark.parametrize("size,scale", [(40.0, None), (1e-4, 1e4 * 128 ** -0.5), (1.0, 1e-3),
                                        (1e4, 1e-4 * 128 ** -0.5)])
def test_scores_of_any_size(size, scale):
    """One token takes nearly all the weight; queries far from 1; nearly equal weights."""
    c = Cache([333, 50], 2, 128, 16, True, seed=13)
    q = randn(2, 4, 128, seed=14, dtype=FP32).mul(size).to(BF16)
    note(f"scores of size {size}, scale {scale}")
    o = K.kronq_cache_attention(q.to(DEV), *c.dev(), scale=scale)
    torch.cuda.synchronize()
    # scores 40 times larger: so are their roundings, and the weights' with them
    tol = TOL + (40 * 4 * 2.0 ** -11 if size == 40.0 else 0.0)
    assert rel_frob(f64(o), c.ref(f64(q), np.arange(3), scale)) < tol


def test_value_scales_side_by_side():
    """Value rows of very different sizes, small before large and large before small, and zeros."""
    c = Cache([400], 1, 128, 16, True, seed=15)
    size = np.exp2(np.concatenate((np.linspace(-30, 10, 200), np.linspace(10, -30, 200))))
    v = (f64(c.v) * size[:, None, None]).astype(np.float32)
    v[::7] = 0
    v = torch.from_numpy(v).to(BF16)
    slots = [int(c.table[0, t // 16]) * 16 + t % 16 for t in range(400)]
    K.kronq_cache_append(c.k.to(DEV), v.to(DEV), torch.tensor(slots, dtype=torch.int64, device=DEV),
                         c.codes, c.params)
    c.held[1] = O.cache_grid(f64(v), True)[3] @ (O.hadamard(128) / np.sqrt(128))
    q = randn(400, 2, 128, seed=16)
    note("value scales side by side")
    o = K.kronq_cache_attention(q.to(DEV), *c.dev(),
                                torch.tensor([0, 400], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    ref = c.ref(f64(q), [0, 400])
    # each row relative to its own size
    row = np.linalg.norm(ref, axis=-1, keepdims=True) + 1e-300
    assert rel_frob(f64(o) / row, ref / row) < TOL


def test_attention_repeats_strides_streams():
    """Bit for bit the same twice, on another stream, with strided q and out, and in a batch with
    other sequences."""
    c = Cache([500, 77, 1200], 4, 128, 64, True, seed=17, wide=3)
    qw = randn(3, 16 + 8, 128, seed=18).to(DEV)
    q = qw[:, 4:20]
    args = c.dev()
    note("attention twice, strided and on another stream")
    a = K.kronq_cache_attention(q, *args)
    wide = torch.full((3, 24, 128), 3.0, dtype=BF16, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        K.kronq_cache_attention(q.contiguous(), *args, out=wide[:, 4:20])
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    assert torch.equal(wide[:, 4:20], a)
    assert bool((wide[:, :4] == 3).all()) and bool((wide[:, 20:] == 3).all())


def test_captured_decode_follows_the_cache():
    """Append and attention of one decode step in a graph; every replay writes the next slot and
    sees one token more, and equals the eager step."""
    c = Cache([60, 10], 2, 128, 16, True, seed=19, wide=2, spare=6)
    codes, params, table, lengths = c.dev()
    free = [p for p in range(codes.shape[0]) if p not in set(c.table.flatten().tolist())]
    table[0, 4], table[1, 1] = free[0], free[1]
    heads = 8
    q = torch.zeros(2, heads, 128, dtype=BF16, device=DEV)
    k, v = (torch.zeros(2, 2, 128, dtype=BF16, device=DEV) for _ in range(2))
    slots = torch.zeros(2, dtype=torch.int64, device=DEV)
    out = torch.zeros(2, heads, 128, dtype=BF16, device=DEV)
    ws = torch.empty(K.kronq_workspace_bytes(K.OP_ATTENTION, heads, 128, 2), dtype=torch.uint8,
                     device=DEV)

    def step():
        K.kronq_cache_append(k, v, slots, codes, params)
        K.kronq_cache_attention(q, codes, params, table, lengths, out=out, ws=ws)

    def feed(i):
        q.copy_(randn(2, heads, 128, seed=30 + i))
        k.copy_(randn(2, 2, 128, seed=40 + i)), v.copy_(randn(2, 2, 128, seed=50 + i))
        at = [60 + i, 10 + i]
        slots.copy_(torch.tensor([int(table[b, t // 16]) * 16 + t % 16 for b, t in enumerate(at)]))
        lengths.copy_(torch.tensor([t + 1 for t in at], dtype=torch.int32))

    note("captured decode steps")
    feed(0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(4):
        feed(i)
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.zero_()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and bool(got.any())


def test_long_cache_offsets_pass_32_bits():
    """A cache whose codes take more than 2^32 bytes and whose words pass 2^31: sequences on its
    first and last pages."""
    kv, dim, page = 8, 128, 4096
    pages = (1 << 31) // (kv * 2 * page * dim // 8) + 3
    if torch.cuda.mem_get_info()[0] < pages * kv * 2 * page * (dim // 8 + 1) * 4 * 1.2:
        pytest.skip("not enough free memory")
    codes = torch.zeros(pages, kv, 2, page * dim // 8, dtype=torch.int32, device=DEV)
    params = torch.zeros(pages, kv, 2, page, dtype=torch.int32, device=DEV)
    assert codes.numel() > 2 ** 31
    k, v = randn(40, kv, dim, seed=60), randn(40, kv, dim, seed=61)
    slots = np.concatenate((np.arange(20), (pages - 1) * page + np.arange(20)))
    note("a cache past 32 bits")
    K.kronq_cache_append(k.to(DEV), v.to(DEV), torch.from_numpy(slots).to(DEV), codes, params)
    table = torch.tensor([[0], [pages - 1]], dtype=torch.int32, device=DEV)
    q = randn(2, 8, dim, seed=62)
    o = K.kronq_cache_attention(q.to(DEV), codes, params, table,
                                torch.tensor([20, 20], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    h = O.hadamard(dim) / np.sqrt(dim)
    hk, hv = (O.cache_grid(f64(t), True)[3] @ h for t in (k, v))
    ref = np.concatenate([O.causal_attention(f64(q)[b:b + 1], hk[20 * b:20 * b + 20],
                                             hv[20 * b:20 * b + 20], dim ** -0.5) for b in (0, 1)])
    assert rel_frob(f64(o), ref) < TOL
