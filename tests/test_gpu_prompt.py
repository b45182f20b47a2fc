"""Attention of whole prompts over themselves against its plain 64-bit form."""
import numpy as np
import pytest
import torch

import paper_2607_22586_amd as mm
from prompts import attention, spans

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def inputs(B, Hq, Hkv, T, d, seed, layout="heads", scale=1.5):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def one(H, s=1.0):
        x = s * torch.randn((B, H, T, d), generator=g, device=DEV)
        if layout == "tokens":                     # [B, T, H, d] as a projection leaves it
            return x.bfloat16().transpose(1, 2).contiguous().transpose(1, 2)
        if layout == "gaps":                       # rows of a larger tensor
            big = torch.full((B, H + 1, T + 3, d + 8), float("nan"), device=DEV, dtype=torch.bfloat16)
            big[:, 1:, 2:T + 2, :d] = x.bfloat16()
            return big[:, 1:, 2:T + 2, :d]
        return x.bfloat16()
    return one(Hq, scale), one(Hkv), one(Hkv)


def int32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def check(got, q, k, v, starts=None, causal=True, lse=None):
    out, tol, want, ltol = attention(q, k, v, starts, causal)
    here = ~np.isnan(out)
    got = got.cpu().double().numpy()
    assert np.isfinite(got[here]).all()
    err = np.abs(got - out)[here]
    assert (err <= tol[here]).all(), (err / tol[here]).max()
    if lse is not None:
        here = ~np.isnan(want)
        err = np.abs(lse.cpu().double().numpy() - want)[here]
        assert (err <= ltol[here]).all(), (err / ltol[here]).max()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("B,Hq,Hkv,T", [(1, 1, 1, 1), (2, 3, 1, 2), (1, 7, 1, 17), (2, 4, 4, 63), (1, 2, 2, 64),
                                        (3, 4, 2, 65), (1, 28, 4, 129), (1, 5, 1, 200), (1, 1, 1, 513),
                                        (2, 16, 2, 300), (1, 2, 1, 1000), (1, 130, 1, 9)])
def test_batches(d, causal, B, Hq, Hkv, T):
    q, k, v = inputs(B, Hq, Hkv, T, d, T)
    out, lse = mm.prompt_attention(q, k, v, causal=causal, with_lse=True)
    check(out, q, k, v, None, causal, lse)
    assert torch.equal(out, mm.prompt_attention(q, k, v, causal=causal))


CUTS = [[0, 1], [0, 300], [0, 0, 1, 1, 2, 300, 300], [0, 100, 200, 300], [0, 64, 128, 192, 256, 300],
        [0, 63, 64, 65, 127, 128, 129, 300], [5, 250], [7, 7, 7], [0, 299], [120, 121, 122, 300], [299, 300],
        list(range(0, 301, 3)), [0, 1, 299, 300], list(range(301)), [0] * 300 + [300], [3] + [150] * 700 + [290]]


@pytest.mark.parametrize("d,Hq,Hkv", [(64, 1, 1), (64, 16, 2), (128, 7, 1), (128, 2, 2)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("cuts", CUTS, ids=range(len(CUTS)))
def test_packed(d, Hq, Hkv, causal, cuts):
    """Sequences of any length, empty ones too; rows in none keep what they held."""
    T = 300
    q, k, v = inputs(1, Hq, Hkv, T, d, len(cuts), "tokens")
    out = torch.full_like(q, 7.0)
    lse = torch.full((1, Hq, T), 7.0, device=DEV)
    mm.prompt_attention(q, k, v, starts=int32(cuts), causal=causal, out=out, lse=lse)
    check(out, q, k, v, cuts, causal, lse)
    inside = torch.zeros(T, dtype=torch.bool, device=DEV)
    for lo, hi in spans(cuts, T):
        inside[lo:hi] = True
    assert bool((out[:, :, ~inside] == 7.0).all()) and bool((lse[:, :, ~inside] == 7.0).all())


@pytest.mark.parametrize("d,Hq,Hkv", [(64, 2, 2), (128, 4, 1)])
@pytest.mark.parametrize("kind", range(5))
def test_many_sequences(d, Hq, Hkv, kind):
    """More starts than threads look at: short sequences, empty ones among them, many at one token or at both ends."""
    T = 1500
    rng = np.random.RandomState(kind)
    cuts = [list(range(0, T + 1)) + [T] * 700, [0] * 2000 + list(range(0, T, 2)) + [T],
            [5] + sorted(rng.randint(5, 1400, 2500).tolist()) + [1400],
            sorted(rng.randint(0, T, 1100).tolist()) + [T] * 3000,
            [0, 700] + [700] * 4000 + [701, 1490]][kind]
    q, k, v = inputs(1, Hq, Hkv, T, d, kind, "tokens")
    for causal in (True, False):
        out = torch.full_like(q, 7.0)
        mm.prompt_attention(q, k, v, starts=int32(cuts), causal=causal, out=out)
        check(out, q, k, v, cuts, causal)
        assert bool((out[:, :, :cuts[0]] == 7.0).all()) and bool((out[:, :, cuts[-1]:] == 7.0).all())


@pytest.mark.parametrize("layout", ["tokens", "gaps"])
@pytest.mark.parametrize("d", [64, 128])
def test_strides(layout, d):
    q, k, v = inputs(2, 6, 2, 150, d, 3, layout)
    out = mm.prompt_attention(q, k, v)
    check(out, q, k, v)
    big = torch.full((2, 150, 9, d + 16), 3.0, device=DEV, dtype=torch.bfloat16)
    got = mm.prompt_attention(q, k, v, out=big[:, :, 1:7, 8:d + 8].transpose(1, 2))
    assert torch.equal(got, out)
    big[:, :, 1:7, 8:d + 8] = 3.0
    assert bool((big == 3.0).all())
    # K and V of one row for all batches
    got = mm.prompt_attention(q, k[:1].expand(2, -1, -1, -1), v[:1].expand(2, -1, -1, -1))
    check(got, q, k[:1].expand(2, -1, -1, -1), v[:1].expand(2, -1, -1, -1))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_infinities_and_nan_stay_with_the_rows_that_see_them(d, causal):
    """Padding and other sequences may hold anything; a row that sees a NaN is NaN, an infinity of V infinite."""
    T, cuts = 333, [3, 40, 41, 170, 300]
    q, k, v = inputs(1, 4, 2, T, d, 11)
    clean = mm.prompt_attention(q, k, v, starts=int32(cuts), causal=causal)
    for t, x in ((0, float("nan")), (2, float("inf")), (300, float("nan")), (332, -float("inf"))):
        k[:, :, t] = x
        v[:, :, t] = x
        q[:, :, t] = x
    got = mm.prompt_attention(q, k, v, starts=int32(cuts), causal=causal)
    assert torch.equal(got[:, :, 3:300], clean[:, :, 3:300])
    # key 100 of the sequence 41 .. 170, in single dims of V
    v[:, 0, 100, 5] = float("nan")
    v[:, 1, 100, d - 1] = float("inf")
    v[:, 1, 101, d - 2] = -float("inf")
    got = mm.prompt_attention(q, k, v, starts=int32(cuts), causal=causal)
    first = 100 if causal else 41
    same = torch.ones_like(got, dtype=torch.bool)
    same[:, :2, first:170, 5] = False
    same[:, 2:, first:170, d - 1] = False
    same[:, 2:, (101 if causal else 41):170, d - 2] = False
    same[:, :, :3] = same[:, :, 300:] = False
    assert torch.equal(got[same], clean[same])
    assert bool(got[:, :2, first:170, 5].isnan().all())
    assert bool((got[:, 2:, first:170, d - 1] == float("inf")).all())
    assert bool((got[:, 2:, (101 if causal else 41):170, d - 2] == -float("inf")).all())
    # a NaN key
    k[:, 0, 200, 0] = float("nan")
    got = mm.prompt_attention(q, k, v, starts=int32(cuts), causal=causal)
    first = 200 if causal else 170
    assert bool(got[:, :2, first:300].isnan().all())
    assert torch.equal(got[:, :2, 170:first], clean[:, :2, 170:first])
    assert torch.equal(got[:, 2:, 170:300], clean[:, 2:, 170:300])


@pytest.mark.parametrize("d", [64, 128])
def test_large_logits_and_growing_maxima(d):
    """Logits to thousands, the maximum late, early, or at every key."""
    T = 400
    for kind in range(3):
        q, k, v = inputs(1, 2, 1, T, d, 5 + kind)
        ramp = torch.linspace(-30, 30, T, device=DEV)
        ramp = (ramp, -ramp, ramp * (torch.arange(T, device=DEV) % 2 * 2 - 1))[kind]
        k = (k.float() + ramp[:, None] * 2).bfloat16()
        q = (q.float() * 4 + 3).bfloat16()
        out, lse = mm.prompt_attention(q, k, v, with_lse=True)
        check(out, q, k, v, lse=lse)
    v = v * 2.0 ** 110
    check(mm.prompt_attention(q, k, v), q, k, v)


def test_a_long_row_key_by_key():
    """All but e^-32 of each query's weight on its own key: none of a long prompt's is left out or counted twice.

    Key t is its 13 bits as -1 and 1, the query 128 times them, so that a key j bits away has e^(-32 j) times the
    weight: together less than 13 e^-32 1.001 < 1.7e-13, of values at most 12 away (a value may be 0): 2.1e-12,
    beside the rounding of the result."""
    T, d = 5000, 64
    k = torch.zeros((1, 1, T, d), device=DEV)
    bits = (torch.arange(T, device=DEV)[:, None] >> torch.arange(13, device=DEV)) & 1
    k[0, 0, :, :13] = (bits * 2 - 1).float()
    q = 8 * 16 * k.expand(1, 2, -1, -1)            # the logit of key t at itself is 13 * 16, at others 32 less or more
    v = torch.randn((1, 1, T, d), device=DEV)
    q, k, v = q.bfloat16(), k.bfloat16(), v.bfloat16()
    out = mm.prompt_attention(q, k, v, causal=False)
    assert float(v.abs().max()) <= 6
    assert bool(((out[0].double() - v[0].double()).abs() <= 2.0 ** -8 * v[0].double().abs() + 2.1e-12).all())


@pytest.mark.parametrize("d,Hq,Hkv,T", [(64, 3, 3, 700), (64, 9, 3, 2500), (128, 3, 1, 1500), (128, 28, 4, 2049),
                                        (128, 9, 9, 8200), (128, 10, 1, 8200)])
@pytest.mark.parametrize("causal", [True, False])
def test_as_in_fp32(d, Hq, Hkv, T, causal):
    """Longer sequences, of each launch shape, against the same formula in fp32 on the GPU: its own error, of sums
    over T rows, is below the bound that the 64-bit form has for the kernel's (2 T u_fp32 beside bf16 roundings)."""
    q, k, v = inputs(1, Hq, Hkv, T, d, T, "tokens")
    out, lse = mm.prompt_attention(q, k, v, causal=causal, with_lse=True)
    t = torch.arange(T, device=DEV)
    for h in range(Hq):
        c = h // (Hq // Hkv)
        kk, vv = k[0, c].float(), v[0, c].float()
        x = q[0, h].float() @ kk.t().contiguous() * d ** -0.5
        size = float((q[0, h].float().abs() @ kk.abs().t().contiguous()).max()) * d ** -0.5
        if causal:
            x = x.masked_fill(t > t[:, None], -float("inf"))
        p = torch.softmax(x, -1)
        want = p @ vv
        rel = 4 * ((d + 4) * 2.0 ** -24 * size + 2.0 ** -23) + 4 * T * 2.0 ** -24
        bound = 2.0 ** -8 * want.abs() + (2.0 ** -8 + rel) * (p @ vv.abs())
        assert bool(((out[0, h].float() - want).abs() <= bound).all())
        assert float((lse[0, h] - torch.logsumexp(x, -1)).abs().max()) <= rel + 2.0 ** -22 * (size + 40)


@pytest.mark.parametrize("d,Hq,Hkv", [(64, 4, 4), (128, 7, 1), (64, 2, 2)])
@pytest.mark.parametrize("cuts", [[0, 700, 1500], [3, 900, 1111, 1112, 1130, 1490], [0, 600, 1210, 1500], [100, 1400],
                                  [0, 1, 1499, 1500]])
def test_long_packed_sequences(d, Hq, Hkv, cuts):
    """Sequences that end within a row tile beside long ones, whose rows other workgroups may have."""
    T = 1500
    q, k, v = inputs(1, Hq, Hkv, T, d, len(cuts) + d, "tokens")
    for causal in (True, False):
        out = torch.full_like(q, 7.0)
        lse = torch.full((1, Hq, T), 7.0, device=DEV)
        mm.prompt_attention(q, k, v, starts=int32(cuts[:2] + cuts[1:]), causal=causal, out=out, lse=lse)
        check(out, q, k, v, cuts, causal, lse)
        inside = torch.zeros(T, dtype=torch.bool, device=DEV)
        inside[cuts[0]:cuts[-1]] = True
        assert bool((out[:, :, ~inside] == 7.0).all()) and bool((lse[:, :, ~inside] == 7.0).all())
        # (fewer sequences on average: two workgroups for a row tile)
        if len(cuts) <= 3:
            again = mm.prompt_attention(q, k, v, starts=int32(cuts), causal=causal)
            check(again, q, k, v, cuts, causal)


def test_rows_behind_four_gib():
    """Strides that put the last tokens past 4 GiB."""
    T, H, d = 70, 2, 64
    step = (1 << 32) // 2 // 64 + 8                # elements: token 64 starts past 4 GiB
    base = torch.empty(T * step, dtype=torch.bfloat16, device=DEV)
    at = base.as_strided((1, H, T, d), (0, d, step, 1))
    q, k, v = inputs(1, H, H, T, d, 8)
    want = mm.prompt_attention(q, k, v)
    at.copy_(k)
    assert torch.equal(mm.prompt_attention(q, at, v), want)
    at.copy_(v)
    assert torch.equal(mm.prompt_attention(q, k, at), want)
    at.copy_(q)
    assert torch.equal(mm.prompt_attention(at, k, v, out=torch.empty_like(q)), want)


def test_captured_on_another_stream():
    q, k, v = inputs(1, 8, 2, 260, 128, 4)
    starts = int32([0, 31, 200, 260])
    out, stream, graph = torch.empty_like(q), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        mm.prompt_attention(q, k, v, starts=starts, out=out)
    for turn in range(3):
        q.copy_(inputs(1, 8, 2, 260, 128, 20 + turn)[0])
        starts.copy_(int32([turn, 30 + turn, 30 + turn, 260]))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check(out, q, k, v, starts.tolist())
        assert bool((out[:, :, :turn] == 0).all())


def test_prompt_written_selected_and_decoded():
    """A prompt's attention, then its rows cached and a further token: the chunk's attention goes on where it ended."""
    B, Hq, Hkv, T, d = 2, 8, 2, 150, 64
    q, k, v = inputs(B, Hq, Hkv, T, d, 6)
    out = mm.prompt_attention(q, k, v)
    cache = mm.PagedCache.empty(B, Hkv, T, d)
    mm.cache_write(cache, k, v)
    lens = torch.full((B, Hkv), T, dtype=torch.int32, device=DEV)
    tail = mm.chunk_attention(q[:, :, -5:], cache, lens)
    full = attention(q, k, v)
    assert (np.abs(tail.cpu().double().numpy() - full[0][:, :, -5:]) <= full[1][:, :, -5:]).all()
    check(out, q, k, v)
