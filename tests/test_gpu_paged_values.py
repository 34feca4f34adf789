"""Values of the paged-pool operators where their types end."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF16, FP16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
DEV = "cuda"


def _coop():
    import paper_2311_00591_amd as coop
    return coop


def _announce(label):
    print(f"[gpu case] paged: {label}", flush=True)
    sys.stdout.flush()


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_cache_write_stores_the_quotients_bytes(dtype):
    """Byte for byte x / scale in 32 bits, limited and rounded: signed zeros,
    numbers that come to zero, and scales past the usual ones (2^-60 to 2^15, a
    mantissa that is not all ones), which are divided by another way."""
    coop = _coop()
    _announce(f"write, bytes of quotients, {dtype}")
    scales = torch.tensor([1.0, 0.013, -0.5, 2.0**-60, 2.0**60, 2.0**-61, 2.0**61, 2.0**-70,
                           2.0**70, 2.0 - 2.0**-23, 2.0**-100, 3.0e38, 2.0**15, 32767.0, 3.0, 2.0**17])
    heads, dim, tokens = len(scales), 64, 40
    g = torch.Generator().manual_seed(3)
    # numbers around what e4m3 holds, times the scale, where the type reaches that far
    x = torch.randn((tokens, heads, dim), generator=g)
    x = x * torch.exp2(torch.randint(-14, 10, x.shape, generator=g).float())
    x = x * scales[:, None]
    x[0, :, :] = 0.0
    x[1, :, :] = -0.0
    tiny = torch.finfo(dtype).smallest_normal
    x[2] = torch.linspace(-2 * tiny, 2 * tiny, dim)  # the type's smallest
    x[3] = 2.0**-12 * scales[:, None] * torch.linspace(-1, 1, dim)  # below e4m3's smallest
    x = x.to(dtype)
    kc, vc = (torch.full((5, 8, heads, dim), 0x55, dtype=torch.uint8, device=DEV).view(E4M3) for _ in "kv")
    coop.cache_write(x.to(DEV), -x.to(DEV), torch.arange(tokens, device=DEV), kc, vc,
                     k_scale=scales.to(DEV), v_scale=scales.to(DEV))
    for cache, rows in ((kc, x), (vc, -x)):
        want = (rows.float() / scales[:, None]).clamp(-448, 448).to(E4M3).view(torch.uint8)
        got = cache.view(torch.uint8).cpu().view(tokens, heads, dim)
        bad = (got != want).nonzero()
        assert len(bad) == 0, [(rows[tuple(i)].item(), scales[i[1]].item(), hex(got[tuple(i)]),
                                hex(want[tuple(i)])) for i in bad[:5]]


@pytest.mark.parametrize("tokens, requests", [(1, 64), (16, 64), (64, 16)])
@pytest.mark.parametrize("dtype", [FP16, BF16])
def test_tree_attention_keeps_weights_far_below_the_largest(tokens, requests, dtype):
    """The first key's score is far above all others, and its value is zero:
    what is left is the sum of thousands of weights of about 2^-23.4 each.

    Bound, with u half a step of the type, A = sum_j w_j |v_j| over n keys (all
    values here are at least zero, so A is the output), dim 64:
      the result's and the weights' rounding           2 u A
      scores of error d = 2^-24 (68 S + 4 s) with S = s = 16.3        2 d A
      32-bit sums over n <= 2112 terms, twice           2.25 n 2^-24 A
      e^x                                               2^-21 A
    and for fp16, whose step below 2^-14 is 2^-24 throughout: the largest
    weight is taken as 2^7, so 2^-25 2^-7 for each key's weight in units of the
    largest, and 2^-25 for a result below 2^-14."""
    coop = _coop()
    _announce(f"attention, small weights, {requests} x {tokens}, {dtype}")
    n, page, dim, heads, group = 2048, 16, 64, 8, 4 if tokens > 1 else 1
    g = torch.Generator().manual_seed(tokens)
    k_cache = torch.zeros((n // page, page, heads, dim))
    v_cache = torch.rand(k_cache.shape, generator=g) + 0.5
    k_cache[0, 0, :, 0] = 4.0625
    v_cache[0, 0] = 0
    total = tokens * requests
    q, k = torch.zeros((total, heads * group, dim)), torch.zeros((total, heads, dim))
    q[:, :, 0] = 4.0
    v = torch.rand((total, heads, dim), generator=g) + 0.5
    q, k, v, k_cache, v_cache = (t.to(DEV, dtype) for t in (q, k, v, k_cache, v_cache))
    table = torch.arange(n // page, dtype=torch.int32, device=DEV).repeat(requests, 1)
    lengths = torch.full((requests,), n, dtype=torch.int64, device=DEV)
    offsets = torch.arange(requests + 1, device=DEV) * tokens
    got = coop.tree_attention(q, k, v, k_cache, v_cache, table, lengths, offsets, scale=1.0)
    score = 4.0 * 4.0625
    w = np.exp(-score)  # of every key but the first
    cached = v_cache.double().cpu().numpy().reshape(n, heads, dim).sum(0)
    own = v.double().cpu().numpy().reshape(requests, tokens, heads, dim).cumsum(1)
    seen = (n - 1 + np.arange(1, tokens + 1))[None, :, None, None]
    want = (cached + own) * w / (1 + seen * w)
    u, d = torch.finfo(dtype).eps / 2, 2.0**-24 * (68 + 4) * score
    tol = (2 * u + 2 * d + 2.25 * seen * 2.0**-24 + 2.0**-21) * want
    if dtype == FP16:
        tol = tol + 2.0**-32 * (cached + own) + 2.0**-25
    want, tol = (np.repeat(x, group, axis=2) for x in (want, tol))
    off = np.abs(got.double().cpu().numpy().reshape(want.shape) - want)
    worst = (off / tol).max()
    print(f"  worst error {worst:.3f} of what rounding allows", flush=True)
    assert worst <= 1
