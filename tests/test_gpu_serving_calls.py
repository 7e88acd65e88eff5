"""Calls of the serving operators that their documentation allows and that lie off the beaten path:
sequences without new tokens, no sequences at all, sizes at the limits, activations at both ends of
fp32's range, sums that add up the roundings of a group. Through the C ABI against the float64 oracle,
with the tolerances of the operators' own tests where nothing else is derived.
"""
import ctypes

import numpy as np
import pytest
import torch

import oracle as O
from gpu_util import DEV, note, rel_frob
from paper_2607_07964_amd import kronq as K
from test_gpu_cache import TOL as TOL_ATTENTION
from test_gpu_cache import Cache, f64, randn
from test_gpu_served import BF16, FP32, TOL, Layer, rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    K.load()
    assert torch.cuda.is_available(), "GPU tests need an MI355X"


def attention_call(q, c, out, n_tokens, starts=None, most=1, flags=1, n_seqs=None):
    """kronq_cache_attention as C has it, with a workspace of just the bytes it asks for."""
    codes, params, table, lengths = c.dev()
    heads, dim = q.shape[1:]
    ws = torch.empty(K.kronq_workspace_bytes(K.OP_ATTENTION, heads, dim, n_tokens),
                     dtype=torch.uint8, device=DEV)
    ptr = lambda t: ctypes.c_void_p(None if t is None else t.data_ptr())  # noqa: E731
    rc = K.load().kronq_cache_attention(
        ptr(q), heads * dim, n_tokens, heads, c.kv, dim, ptr(codes), ptr(params), codes.shape[0],
        c.page, ptr(table), table.shape[1], table.shape[1], ptr(lengths),
        table.shape[0] if n_seqs is None else n_seqs, ptr(starts), most, dim ** -0.5, flags, ptr(out),
        heads * dim, ptr(ws), ws.numel(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    return rc


@pytest.mark.parametrize("lengths,tokens", [([40, 90, 33, 70], 2), ([900, 1500, 700], 1),
                                            ([1300, 40, 2000, 1, 999], 3)])
def test_attention_of_fewer_tokens_than_sequences(lengths, tokens):
    """Without starts, sequences from n_tokens on have no new token: neither rows of q behind the last
    one are read nor rows of out written, undivided and with the tokens split over workgroups."""
    c = Cache(lengths, 2, 128, 16, True, seed=31)
    q = randn(len(lengths) + 2, 8, 128, seed=32)
    q[tokens:] = float("nan")
    out = torch.full((len(lengths) + 2, 8, 128), 3.0, dtype=BF16, device=DEV)
    note(f"attention of {tokens} tokens over sequences {lengths}")
    assert attention_call(q.to(DEV), c, out, tokens) == 0
    ref = c.ref(f64(q[:tokens]), np.minimum(np.arange(len(lengths) + 1), tokens))
    assert rel_frob(f64(out[:tokens]), ref) < TOL_ATTENTION
    assert bool((out[tokens:] == 3).all())


@pytest.mark.parametrize("tokens,heads,dim", [(1, 1, 64), (7, 4, 128), (70000, 2, 64)])
def test_attention_without_sequences(tokens, heads, dim):
    """Every token is one of no sequence: zeros where they are asked for, and nothing otherwise."""
    codes, params = K.kronq_cache_empty(1, 1, dim, 16, DEV)
    q = torch.randn(tokens, heads, dim, dtype=BF16, device=DEV)
    rows = torch.full((tokens + 1, heads * dim + 3), 3.0, dtype=BF16, device=DEV)
    nul, ptr = ctypes.c_void_p(0), lambda t: ctypes.c_void_p(t.data_ptr())
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    note(f"attention of {tokens} tokens without sequences")
    for flags, want in ((1, 3.0), (3, 0.0)):
        assert K.load().kronq_cache_attention(
            ptr(q), heads * dim, tokens, heads, 1, dim, ptr(codes), ptr(params), 1, 16, nul, 0, 0, nul,
            0, nul, 1, 0.1, flags, ptr(rows), heads * dim + 3, nul, 0, stream) == 0
        torch.cuda.synchronize()
        assert bool((rows[:tokens, :heads * dim] == want).all())
        assert bool((rows[:, heads * dim:] == 3).all()) and bool((rows[tokens] == 3).all())
    table, none = torch.zeros(0, 4, dtype=torch.int32, device=DEV), torch.zeros(0, dtype=torch.int32,
                                                                              device=DEV)
    starts = torch.zeros(1, dtype=torch.int32, device=DEV)
    torch.full_like(q, float("nan"))  # (what the allocator hands out next is not zero)
    out = K.kronq_cache_attention(q, codes, params, table, none, starts)
    torch.cuda.synchronize()
    assert out.shape == q.shape and not bool(out.any())


def whole_numbers(d_out, d_in, bits, experts=1):
    """A layer without transforms whose scales are one power of two: with small whole activations every
    product and every sum is a whole number times it, so that only the result is rounded."""
    la = Layer(d_out, d_in, bits, 128, 0, experts=experts, bias=False)
    la.scales[:], la.mul_in[:], la.mul_out[:] = 2.0 ** -7, 1.0, 1.0
    la.device()
    return la


@pytest.mark.parametrize("bits", [2, 3, 4, 8])
@pytest.mark.parametrize("rows,d_out,d_in", [(300, 200, 4096), (700, 513, 2176), (257, 64, 128)])
def test_whole_numbers_are_rounded_once(bits, rows, d_out, d_in):
    """Many rows, few items, columns split over many workers: the sums are exact in fp32 (below 2^24
    of their unit), so that the result is the bf16 value next to them, bit for bit."""
    la = whole_numbers(d_out, d_in, bits)
    x = torch.randint(-8, 9, (rows, d_in), generator=torch.Generator().manual_seed(rows)).to(BF16)
    note(f"whole numbers bits={bits} rows={rows} {d_out}x{d_in}")
    y = K.kronq_online_linear(*la.args, None, None, None, None, x.to(DEV), flags=0)
    torch.cuda.synchronize()
    ref = torch.from_numpy(la.ref(f64(x)))
    assert float(ref.abs().max()) * 2 ** 7 < 2 ** 24
    assert torch.equal(y.cpu(), ref.to(FP32).to(BF16))


@pytest.mark.parametrize("bits", [3, 4, 8])
@pytest.mark.parametrize("experts,rows", [(1, 300), (3, 400)])
def test_weights_of_both_signs_cancel(bits, experts, rows):
    """As many weights s 2^k as -s 2^k in every group, and activations that are all alike: the
    definition gives zero, and so does any rounding of s and of the weights that is the same for both
    signs, but for the sums' own. An offset that the weights of a group share would add up."""
    la = Layer(160, 1024, bits, 128, 0, experts=experts, bias=False)
    r = np.random.default_rng(bits)
    k = np.exp2(r.integers(0, bits - 2, (experts, 160, 8, 64))).astype(np.int64)
    whole = r.permuted(np.concatenate((k, -k), -1), axis=-1)
    zeros = r.integers(2 ** (bits - 2), 3 * 2 ** (bits - 2) + 1, (experts, 160, 8))  # |whole| from both ends
    assert np.abs(whole).max() <= 2 ** (bits - 2)
    la.zeros, la.codes = zeros.astype(np.float32), (whole + zeros[..., None]).astype(np.uint8)
    whole, la.codes = (t.reshape(experts, 160, 1024) for t in (whole, la.codes))
    assert np.array_equal(la.codes - np.repeat(zeros, 128, -1), whole)
    la.mul_in[:], la.mul_out[:] = 1.0, 1.0
    la.device()
    x = torch.full((rows, 1024), 2.625, dtype=BF16, device=DEV)
    note(f"weights that cancel bits={bits} experts={experts}")
    if experts == 1:
        y = K.kronq_online_linear(*la.args, None, None, None, None, x, flags=0)
    else:
        offsets = torch.tensor([0, 100, 290, 400], dtype=torch.int32, device=DEV)
        y = K.kronq_online_grouped(*la.args, None, None, None, None, x, offsets, flags=0)
    torch.cuda.synchronize()
    # A product s 2^k 21 2^j has 11 + 5 bits beside 2^k, a partial sum of a group up to 64 of the largest
    # more: 11 + 5 + 6 + 5 bits with 8-bit codes (k <= 5), beyond fp32's 24. Each of 1024 additions is
    # then off by at most 2^-23 of a partial sum (cut off or rounded), which is at most half of the sum
    # of all |w x| of a group (as much of it is positive as negative). The shared offset of s and z s
    # rounded apart is up to 2^-11 * 128 s for each of 128 weights of 8 groups, some hundred times this.
    half_sum = (np.abs(whole).reshape(experts, 160, 8, 128).sum(-1) / 2 * la.scales * 2.625).max(-1)
    bound = 1024 * 2.0 ** -23 * half_sum.max(0)
    assert np.all(np.abs(f64(y)) <= bound)


@pytest.mark.parametrize("bits", [2, 3, 4, 8])
@pytest.mark.parametrize("experts,rows", [(1, 300), (3, 400)])
@pytest.mark.parametrize("mean", [1.0, 3.0])
def test_activations_of_nonzero_mean(bits, experts, rows, mean):
    """Many rows (the table of fp16 scales). A scale is off by 2^-11 for all of its group, a weight and
    an activation by 2^-11 each, independently of the next group's or column's: 3 * 2^-11 beside the
    result's 2^-8."""
    la = Layer(224, 2048, bits, 128, 0, experts=experts, bias=False)
    r, top = np.random.default_rng(bits), 2 ** bits - 1  # codes of min-max grids of normal values
    la.codes = np.clip(np.rint(r.normal(top / 2, top / 5.4, la.codes.shape)), 0, top).astype(np.uint8)
    la.zeros = np.clip(np.rint(r.normal(top / 2, 0.3, la.zeros.shape)), 0, top).astype(np.float32)
    la.mul_in[:] = 1.0
    la.device()
    x = (rows_of(rows, 2048, FP32) + mean).to(BF16)
    note(f"activations of mean {mean} bits={bits} experts={experts}")
    if experts == 1:
        y, cuts = K.kronq_online_linear(*la.one(), x.to(DEV), flags=0), [0, rows]
    else:
        cuts = [0, 100, 290, 400]
        y = K.kronq_online_grouped(*la.args, *la.factors, x.to(DEV),
                                   torch.tensor(cuts, dtype=torch.int32, device=DEV), flags=0)
    torch.cuda.synchronize()
    ref = np.concatenate([la.ref(f64(x)[a:b], e=e) for e, (a, b) in enumerate(zip(cuts, cuts[1:]))])
    assert rel_frob(f64(y), ref) < 2.0 ** -8 + 3 * 2.0 ** -11


@pytest.mark.parametrize("bits", [2, 3, 4, 8])
def test_many_rows_with_zeros_outside_the_codes(bits):
    la = Layer(96, 256, bits, 128, 0)
    la.zeros = np.random.default_rng(bits).integers(-1024, 1024, la.zeros.shape).astype(np.float32)
    la.zeros[0, :4, 0] = -1024, 1023, -1023, 1022
    la.device()
    x = rows_of(300, 256, BF16) + 0.5
    note(f"many rows, zeros far outside bits={bits}")
    y = K.kronq_online_linear(*la.one(), x.to(DEV), bias=la.bias_d[0], flags=0)
    torch.cuda.synchronize()
    assert rel_frob(f64(y), la.ref(f64(x))) < TOL[BF16]


@pytest.mark.parametrize("bits", [2, 3, 4, 8])
def test_many_rows_with_scales_of_many_sizes(bits):
    """Groups of a row whose scales lie up to 2^14 apart, rows of W of different sizes: activations in
    one group of columns at a time, so that each group's weights are seen by themselves."""
    la = Layer(192, 1024, bits, 128, 0, bias=False)
    size = np.exp2([0.0, -3, -6, -8, -10, -12, -13, -13])
    la.scales = (np.random.default_rng(1).uniform(1, 2, la.scales.shape) * size
                 * np.exp2(np.arange(192) % 40 - 20.0)[:, None]).astype(np.float32)
    la.mul_in[:], la.mul_out[:] = 1.0, 1.0
    la.device()
    x = torch.zeros(8 * 40, 1024)
    for g in range(8):
        x[40 * g:40 * g + 40, 128 * g:128 * g + 128] = rows_of(40, 128, FP32, seed=g) + 0.5
    x = x.to(BF16)
    note(f"many rows, scales of many sizes bits={bits}")
    y = K.kronq_online_linear(*la.one(), x.to(DEV), flags=0)
    torch.cuda.synchronize()
    ref = la.ref(f64(x))
    unit = np.repeat(la.scales[0], 40, axis=1).T  # [row of x, row of W]: the scale of its group
    assert rel_frob(f64(y) / unit, ref / unit) < TOL[BF16]


@pytest.mark.parametrize("exponent", [-112, -104, -93, 105, 116, 122])
@pytest.mark.parametrize("rows", [20, 70, 300])
@pytest.mark.parametrize("flags", [0, K.ROT_IN | K.ROT_OUT])
def test_activations_at_both_ends_of_the_range(exponent, rows, flags):
    """Rows whose largest value lies next to the ends of fp32 (those of 2^4 more and less beside them),
    and weights that bring the results back: as exact as others."""
    la = Layer(256, 512, 4, 128, flags, bias=False)
    la.scales = np.ldexp(la.scales, -exponent * 4 // 5).astype(np.float32)
    la.mul_in, la.mul_out = np.sign(la.mul_in), np.sign(la.mul_out)
    la.device()
    x = rows_of(rows, 512, FP32)
    x /= x.abs().amax(1, keepdim=True)
    x *= torch.exp2(exponent + (torch.arange(rows) % 5).float()[:, None])
    note(f"activations of 2^{exponent} rows={rows} flags={flags}")
    y = K.kronq_online_linear(*la.one(), x.to(DEV), flags=flags, out_dtype=BF16)
    y32 = K.kronq_online_linear(*la.one(), x.to(DEV), flags=flags)
    torch.cuda.synchronize()
    unit = f64(x.abs().amax(1, keepdim=True))
    got, got32, ref = f64(y) / unit, f64(y32) / unit, la.ref(f64(x)) / unit
    if flags:
        # The sums of the transform come before its norm, and with the largest exponent some pass fp32's
        # largest number (22 * 2^126 = 2^130.5): those rows are not finite, as in any fp32 sum. A row
        # goes either way if only a sum on the way may.
        xm = f64(x) * la.mul_in[0]
        over = np.abs(xm @ O.hadamard(512)).max(1) >= 2.0 ** 128
        fine = np.isfinite(got).all(1)
        assert over.any() == (exponent == 122) and np.array_equal(fine, np.isfinite(got32).all(1))
        assert not np.isfinite(got[over]).any() and not np.isfinite(got32[over]).any()
        assert fine.any() and fine[np.abs(xm).sum(1) < 2.0 ** 128].all()
        got, got32, ref = got[fine], got32[fine], ref[fine]
    assert rel_frob(got, ref) < TOL[BF16]
    assert rel_frob(got32, ref) < TOL[FP32]


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("tokens,new", [(2, 1), (3, 1), (5, 5), (8, 1), (8, 8), (33, 33)])
def test_values_whose_codes_are_their_zeros(dim, tokens, new):
    """Channels that hold zero for every token stay zero but for the rounding of fp32 sums, whatever the
    weights are rounded to: the codes' sum and the zeros' sum, each of up to 40 terms of at most 15 of the
    largest scale and weights that add up to one, off by 40 * 2^-24 of that at most, and as much again for
    the changes of reference."""
    r = np.random.default_rng(tokens + dim)
    heads, page = 24, 64
    codes, params = K.kronq_cache_empty(1, 1, dim, page, DEV)
    value = r.integers(0, 16, (page, dim))
    scale = O.round_up_bf16(np.exp(0.3 * r.standard_normal((2, page))))
    zero = r.integers(0, 16, (2, page))
    value[:, 5:20] = zero[1][:, None]
    words = np.stack([O.cache_words(r.integers(0, 16, (page, dim)), 0), O.cache_words(value, 1)])
    codes.copy_(torch.from_numpy(words.view(np.int32))[None, None])
    held = scale.astype(np.float32).view(np.uint32) | zero.astype(np.uint32)
    params.copy_(torch.from_numpy(held.view(np.int32))[None, None])
    q = randn(new, heads, dim, seed=tokens) * 0.2
    starts = torch.tensor([0, new], dtype=torch.int32, device=DEV)
    note(f"values of zero dim={dim} tokens={tokens} new={new}")
    o = K.kronq_cache_attention(q.to(DEV), codes, params, torch.zeros(1, 1, dtype=torch.int32, device=DEV),
                                torch.tensor([tokens], dtype=torch.int32, device=DEV), starts, new,
                                rotate=False)
    torch.cuda.synchronize()
    k = scale[0][:, None] * (codes_of(words[0], dim) - zero[0][:, None])
    v = scale[1][:, None] * (value - zero[1][:, None])
    ref = O.causal_attention(f64(q), k[:tokens, None], v[:tokens, None], dim ** -0.5)
    assert rel_frob(f64(o), ref) < TOL_ATTENTION
    assert np.abs(f64(o)[:, :, 5:20]).max() <= 4 * 40 * 2.0 ** -24 * 15 * scale[1].max()


def codes_of(words, dim):
    """The codes of packed key words."""
    w = words.reshape(-1, dim // 8, 1) >> (4 * np.arange(8, dtype=np.uint32))
    return (w & 15).reshape(-1, dim).astype(np.int64)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,new,at", [(8, 100, 50), (8, 100, 99), (2, 40, 17), (1, 5, 3),
                                          (4, 300, 131)])
@pytest.mark.parametrize("size", [2.0 ** 40, 1e36])
def test_values_of_later_tokens_do_not_reach_earlier_rows(dim, heads, new, at, size):
    """One token's value far above all others: the queries before it are as exact as without it, those
    after it see it."""
    c = Cache([new + 7], 1, dim, 16, True, seed=41)
    v = f64(c.v)
    v[at + 7] *= size
    v = torch.from_numpy(v).to(BF16)
    slots = [int(c.table[0, t // 16]) * 16 + t % 16 for t in range(new + 7)]
    K.kronq_cache_append(c.k.to(DEV), v.to(DEV), torch.tensor(slots, dtype=torch.int64, device=DEV),
                         c.codes, c.params)
    c.held[1] = O.cache_grid(f64(v), True)[3] @ (O.hadamard(dim) / np.sqrt(dim))
    q = randn(new, heads, dim, seed=42)
    note(f"a later token's value dim={dim} heads={heads} new={new} at={at} size={size}")
    o = K.kronq_cache_attention(q.to(DEV), *c.dev(), torch.tensor([0, new], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    ref = c.ref(f64(q), [0, new])
    row = np.linalg.norm(ref, axis=-1, keepdims=True)
    assert rel_frob(f64(o) / row, ref / row) < TOL_ATTENTION


def room_for(gigabytes):
    if torch.cuda.mem_get_info()[0] < gigabytes * 2 ** 30 * 1.1:
        pytest.skip("not enough free memory")


def test_as_many_rows_as_the_limit():
    """2^24 rows: as many workgroups of either side, of 256 threads each, are 2^32 work-items."""
    room_for(22)
    la = whole_numbers(5, 128, 4)
    few = torch.randint(-8, 9, (4099, 128), generator=torch.Generator().manual_seed(1)).to(BF16).to(DEV)
    n = 1 << 24
    x = few.repeat(-(-n // 4099), 1)[:n].contiguous()
    note("2^24 rows of 128")
    y = K.kronq_online_linear(*la.args, None, None, None, None, x, flags=0)
    torch.cuda.synchronize()
    want = torch.from_numpy(la.ref(f64(few))).to(FP32).to(BF16).to(DEV)
    assert torch.equal(y, want.repeat(-(-n // 4099), 1)[:n])
    with pytest.raises(K.KronqError, match="sizes"):
        K.kronq_online_linear(*la.args, None, None, None, None, x[:1].expand(n + 1, 128),
                              torch.empty(1, 5, dtype=BF16, device=DEV).expand(n + 1, 5), flags=0)


def test_rows_of_28_m_past_2_22():
    """Rows of 28 * 32 inputs take workgroups of 1024 threads."""
    room_for(34)
    la = Layer(3, 896, 4, 128, K.ROT_IN)
    few = rows_of(1021, 896, BF16)
    n = (1 << 22) + 300
    x = few.to(DEV).repeat(-(-n // 1021), 1)[:n].contiguous()
    note("rows of 896 past 2^22")
    y = K.kronq_online_linear(*la.one(), x, bias=la.bias_d[0], flags=K.ROT_IN)
    torch.cuda.synchronize()
    ref = la.ref(f64(few))
    for a in (0, 1021 * 2054, 1021 * 4107):  # whole repetitions from the first to the last one
        assert rel_frob(f64(y[a:a + 1021]), ref) < TOL[BF16]
    assert rel_frob(f64(y[1021 * 4108:]), ref[:n - 1021 * 4108]) < TOL[BF16]


def test_append_of_many_rows():
    """Tokens times heads past 2^27, of which some are written: the first and the last ones."""
    room_for(35)
    kv, n = 2048, 65536 + 3
    k = torch.empty(n, kv, 128, dtype=BF16, device=DEV)
    at = [0, 1, 40000, n - 2, n - 1]
    k[at] = randn(len(at), kv, 128, seed=51).to(DEV)
    slots = torch.full((n,), -1, dtype=torch.int64, device=DEV)
    slots[at] = torch.tensor([3, 15, 0, 7, 8], device=DEV)
    codes, params = K.kronq_cache_empty(1, kv, 128, 16, DEV)
    note("append of 2^27 rows")
    K.kronq_cache_append(k, k, slots, codes, params)
    few = K.kronq_cache_empty(1, kv, 128, 16, DEV)
    K.kronq_cache_append(k[at], k[at], slots[at], *few)
    torch.cuda.synchronize()
    assert torch.equal(codes, few[0]) and torch.equal(params, few[1])
    held = O.cache_grid(f64(k[n - 1, :3]), True)
    assert np.array_equal(codes_of(codes[0, :3, 0].cpu().numpy().view(np.uint32).reshape(3, 16, 16)[:, 8],
                                   128), held[0])


def test_attention_of_more_tiles_than_a_grid_dimension():
    """A sequence of 12.8 million rows of one kv head: more tiles than the grid's last dimension holds.
    Only the last queries see tokens."""
    room_for(8)
    c = Cache([40], 1, 64, 16, True, seed=61)
    n, heads = 200_000, 64
    q = torch.full((n, heads, 64), 2.0, dtype=BF16, device=DEV)
    last = randn(40, heads, 64, seed=62)
    q[n - 40:] = last.to(DEV)
    note("attention of 12.8 million rows")
    o = K.kronq_cache_attention(q, *c.dev(), torch.tensor([0, n], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    assert not bool(o[:n - 40].any())
    assert rel_frob(f64(o[n - 40:]), c.ref(f64(last), [0, 40])) < TOL_ATTENTION


def test_decode_of_as_many_sequences_as_the_limit():
    """65535 sequences that share pages, of every length up to 48."""
    c = Cache([48], 1, 64, 16, True, seed=63)
    codes, params, table, _ = c.dev()
    n = 65535
    lengths = (torch.arange(n, device=DEV) % 49).to(torch.int32)
    q = randn(1, 2, 64, seed=64).repeat(n, 1, 1)
    note("decode of 65535 sequences")
    o = K.kronq_cache_attention(q.to(DEV), codes, params, table.expand(n, -1).contiguous(), lengths)
    torch.cuda.synchronize()
    k, v = c.held
    for length in range(49):
        ref = O.causal_attention(f64(q[:1]), k[:length], v[:length], 64 ** -0.5)
        mine = o[length::49]
        assert bool((mine == mine[0]).all())
        assert rel_frob(f64(mine[:1]), ref) < TOL_ATTENTION if length else not bool(mine.any())


def walsh(x):
    """H x / sqrt(d) along the last axis."""
    d = x.shape[-1]
    y, s = x.copy(), 1
    while s < d:
        a = y.reshape(*x.shape[:-1], d // (2 * s), 2, s)
        y = np.concatenate((a[..., :1, :] + a[..., 1:, :], a[..., :1, :] - a[..., 1:, :]), -2).reshape(x.shape)
        s *= 2
    return y / np.sqrt(d)


@pytest.mark.parametrize("rows", [2, 6, 300])
@pytest.mark.parametrize("ydt", [BF16, FP32])
@pytest.mark.parametrize("d_out,d_in,flags", [(24, 32768, K.ROT_IN), (32768, 128, K.ROT_OUT)])
def test_the_largest_sides(rows, ydt, d_out, d_in, flags):
    la = Layer(d_out, d_in, 4, 128, flags)
    x = rows_of(rows, d_in, BF16)
    note(f"{d_out}x{d_in} rows={rows} {ydt}")
    y = K.kronq_online_linear(*la.one(), x.to(DEV), bias=la.bias_d[0], flags=flags, out_dtype=ydt)
    torch.cuda.synchronize()
    w = O.dequantize(la.codes[0], la.scales[0].astype(np.float64), la.zeros[0].astype(np.float64), 128)
    t = f64(x) * la.mul_in[0]
    t = (walsh(t) if flags & K.ROT_IN else t) @ w.T
    ref = (walsh(t) if flags & K.ROT_OUT else t) * la.mul_out[0] + la.bias[0]
    assert rel_frob(f64(y), ref) < TOL[ydt]
