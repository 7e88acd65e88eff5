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
