"""hilo_attention against softmax attention in 64 bits on the same 16-bit inputs.

Tolerance, per element (u = half a step of the dtype, p and v of the row's sum
o = sum p v / sum p): each probability is rounded once before the product
(u sum p |v|), the result once (u |o|); the fp32 logits of up to a few tens are
off by less than 2^-14, as are the exponentials, maxima and sums together
(2^-13 sum p |v|). fp16 probabilities below its normal range round to a
multiple of 2^-24 (half of it per key, against a largest probability of 1 or
more).
"""
import math

import pytest
import torch

from .gpu_helpers import lib_ready

pytestmark = pytest.mark.gpu
TYPES = {"bf16": (torch.bfloat16, 0), "f16": (torch.float16, 2)}


@pytest.fixture(scope="module")
def H():
    return lib_ready()


def offsets(lens, first=0):
    o = [first]
    for n in lens:
        o.append(o[-1] + n)
    return torch.tensor(o, dtype=torch.int32, device="cuda")


def make(lq, lk, heads, kv, hd, dtype="bf16", first=0, spare=0, seed=0, sharp=2.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = TYPES[dtype][0]
    nq, nk = first + sum(lq) + spare, first + sum(lk) + spare
    q = (sharp * torch.randn(nq, heads, hd, generator=g, device="cuda")).to(t)
    k = torch.randn(nk, kv, hd, generator=g, device="cuda").to(t)
    v = torch.randn(nk, kv, hd, generator=g, device="cuda").to(t)
    return q, k, v, offsets(lq, first), offsets(lk, first)


def call(H, q, k, v, cu_q, cu_k, causal=1, out=None, scale=0.0, ws=None, stream=None, fill=float("nan")):
    heads, kv, hd = q.shape[1], k.shape[1], q.shape[2]
    if out is None:
        out = torch.full(q.shape, fill, dtype=q.dtype, device="cuda")
    sh = H.AttnShape(B=cu_q.numel() - 1, heads=heads, kv_heads=kv, head_dim=hd, rows_q=q.shape[0], rows_k=k.shape[0],
                     causal=causal, dtype=0 if q.dtype == torch.bfloat16 else 2, scale=scale, q_row=q.stride(0),
                     q_head=q.stride(1), k_row=k.stride(0), k_head=k.stride(1), v_row=v.stride(0), v_head=v.stride(1),
                     out_row=out.stride(0), out_head=out.stride(1))
    n = H.hilo_attention_workspace_bytes(sh)
    if ws is None:
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    H.hilo_attention(sh, cu_q, cu_k, q, k, v, out, ws, n, stream)
    return out


def reference(q, k, v, cu_q, cu_k, causal, scale=0.0):
    """(o, sum p |v| / sum p, keys) in 64 bits; rows outside the sequences NaN."""
    hd, g = q.shape[2], q.shape[1] // k.shape[1]
    scale = scale or 1 / math.sqrt(hd)
    o = torch.full(q.shape, math.nan, dtype=torch.float64, device="cuda")
    mag = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    cq, ck = cu_q.tolist(), cu_k.tolist()
    for b in range(len(cq) - 1):
        q0, q1, k0, k1 = cq[b], cq[b + 1], ck[b], ck[b + 1]
        if q1 == q0:
            continue
        kk = k[k0:k1].double().repeat_interleave(g, 1).transpose(0, 1)
        vv = v[k0:k1].double().repeat_interleave(g, 1).transpose(0, 1)
        s = (q[q0:q1].double().transpose(0, 1) @ kk.transpose(1, 2)) * scale
        if causal:
            i = torch.arange(q1 - q0, device="cuda")[:, None] + (k1 - k0) - (q1 - q0)
            s = s.masked_fill(torch.arange(k1 - k0, device="cuda") > i, -math.inf)
        if k1 > k0:
            p = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-1e300))
            n = p.sum(-1, keepdim=True).clamp(min=1e-300)
            o[q0:q1] = (p @ vv / n).transpose(0, 1)
            mag[q0:q1] = (p @ vv.abs() / n).transpose(0, 1)
        else:
            o[q0:q1] = 0
    return o, mag, k.shape[0]


def check(got, ref, dtype):
    o, mag, keys = ref
    t = TYPES[dtype][0]
    u = torch.finfo(t).eps / 2
    tol = (u + 2.0 ** -13) * mag + u * o.abs() + (keys * 2.0 ** -25 * 8 if dtype == "f16" else 0.0) + 1e-30
    inside = ~o.isnan()
    assert bool(got[inside].isfinite().all())
    off = ((got.double() - o).abs() / tol)[inside]
    worst = float(off.max()) if off.numel() else 0.0
    assert worst <= 1.0, worst
    assert bool(got[~inside].isnan().all()), "rows outside the sequences were written"


CASES = [
    # lq, lk (None: the same), heads, kv heads, head_dim, causal, dtype
    ([1], None, 1, 1, 64, 1, "bf16"),
    ([1, 2, 127, 128, 129], None, 2, 2, 128, 1, "bf16"),
    ([255, 256, 257, 0, 1, 300], None, 2, 1, 64, 1, "f16"),
    ([333], None, 3, 1, 128, 1, "bf16"),
    ([200, 513], None, 10, 2, 64, 0, "bf16"),
    ([77, 0, 131], None, 14, 2, 128, 1, "f16"),
    ([640], None, 16, 1, 64, 1, "bf16"),
    ([5, 1, 40], None, 128, 1, 128, 1, "bf16"),
    ([9], None, 100, 1, 64, 0, "f16"),
    # chunks over earlier tokens, single tokens, sequences without keys or queries
    ([1, 1, 1, 1], [1, 129, 5000, 64], 8, 2, 128, 1, "bf16"),
    ([1, 0, 3], [0, 17, 0], 4, 4, 64, 0, "bf16"),
    ([100, 17, 1], [1100, 4000, 2], 6, 2, 64, 1, "f16"),
    ([64], [20000], 4, 1, 128, 0, "bf16"),
    ([300, 7], [2048, 2048], 4, 4, 128, 1, "bf16"),
    # more queries than keys: the first ones see none
    ([200, 5, 300], [70, 0, 299], 4, 2, 128, 1, "bf16"),
    # many sequences, in the plan's table and beyond it
    ([3] * 300, [1 + 7 * (i % 40) for i in range(300)], 4, 2, 64, 1, "bf16"),
    ([1 + i % 3 for i in range(1300)], [4 + i % 300 for i in range(1300)], 2, 1, 128, 1, "bf16"),
    # a long sequence among short ones: cut where more jobs than CTAs are there
    ([1] * 100 + [260], [60] * 100 + [9000], 8, 4, 64, 1, "bf16"),
    # fewer jobs than CTAs, dealt out like many: single tokens, one of them over a long cache
    ([1] * 16, [64, 16000, 1, 300] + [70 + 90 * i for i in range(12)], 16, 8, 64, 1, "bf16"),
    ([1] * 45, [12000] + [1 + 13 * i for i in range(44)], 6, 3, 128, 0, "f16"),
    # few sequences, more jobs than the table has, and more than one warp plans
    ([2100], [70], 128, 1, 64, 0, "bf16"),
    ([700, 0, 90], [300, 5, 200], 64, 1, 128, 1, "f16"),
    ([2500], None, 4, 4, 64, 1, "bf16"),
    ([1500, 700], None, 16, 8, 128, 1, "f16"),
    ([1024, 2048], None, 24, 24, 128, 0, "bf16"),
]


@pytest.mark.parametrize("lq,lk,heads,kv,hd,causal,dtype", CASES)
def test_against_64_bits(H, lq, lk, heads, kv, hd, causal, dtype):
    lk = lq if lk is None else lk
    q, k, v, cu_q, cu_k = make(lq, lk, heads, kv, hd, dtype, first=3, spare=5, seed=len(lq) + sum(lk))
    got = call(H, q, k, v, cu_q, cu_k, causal)
    H.hilo_sync_status()
    check(got, reference(q, k, v, cu_q, cu_k, causal), dtype)


@pytest.mark.parametrize("causal", [0, 1])
def test_growing_logits_rescale(H, causal):
    """Keys whose logits rise along the sequence: the running maximum moves at every tile."""
    q, k, v, cu_q, cu_k = make([400], [1500], 4, 2, 128, "bf16", seed=3, sharp=1.0)
    q[:] = q.abs()
    k[:] = k.abs() * torch.linspace(0.05, 1.5, 1500, device="cuda")[:, None, None].to(k.dtype)
    ref = reference(q, k, v, cu_q, cu_k, causal)
    got = call(H, q, k, v, cu_q, cu_k, causal)
    # logits of up to 150: fp32 products of 128 terms are off by up to 150 * 2^-17
    o, mag, n = ref
    check(got, (o, mag * (1 + 150 * 2.0 ** -17 / 2.0 ** -8), n), "bf16")


def test_scale_and_strides(H):
    """q, k and v as columns of one product, a cache ordered by head, out ordered by head; a scale of its own."""
    lq, hd = [130, 61], 64
    q, k, v, cu_q, cu_k = make(lq, lq, 6, 2, hd, "bf16", spare=2, seed=9)
    n = q.shape[0]
    rows = torch.cat([x.reshape(n, -1) for x in (q, k, v)], 1)
    pad = torch.cat([rows, torch.full((n, 8), math.nan, dtype=rows.dtype, device="cuda")], 1)
    fq, fk, fv = (x.unflatten(1, (-1, hd)) for x in pad[:, :-8].split([6 * hd, 2 * hd, 2 * hd], 1))
    ref = reference(q, k, v, cu_q, cu_k, 1, scale=0.3)
    check(call(H, fq, fk, fv, cu_q, cu_k, 1, scale=0.3), ref, "bf16")
    hk, hv = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (k, v))
    store = torch.full((6, n + 1, hd + 8), math.nan, dtype=q.dtype, device="cuda")
    out = store[:, :n, :hd].transpose(0, 1)
    check(call(H, q, hk, hv, cu_q, cu_k, 1, out=out, scale=0.3), ref, "bf16")
    assert bool(store[:, n].isnan().all()) and bool(store[:, :, hd:].isnan().all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("lq,lk,heads", [([300], [300], 2), ([90], [1400], 4), ([200], [450], 12)])
def test_infinities_and_nans_of_unseen_keys(H, dtype, lq, lk, heads):
    """Keys past a query, behind the sequence and of other sequences may hold anything; a query that does see
    an infinite value gets it, and only in its column."""
    q, k, v, cu_q, cu_k = make(lq, lk, heads, 2, 128, dtype, first=2, spare=6, seed=5)
    clean = reference(q, k, v, cu_q, cu_k, 1)
    k[:2], v[:2], k[-6:], v[-6:] = math.nan, math.inf, math.nan, math.nan
    base = call(H, q, k, v, cu_q, cu_k, 1)
    check(base, clean, dtype)
    # the last keys hold infinities and NaNs in a few columns
    n_q, n_k = lq[0], lk[0]
    for back, col, value in ((0, 5, math.inf), (1, 70, math.nan), (37, 9, -math.inf), (64, 127, math.inf)):
        row = 2 + n_k - 1 - back
        v[row, :, col] = value
    k[2 + n_k - 1] = math.nan  # seen by the last query alone
    got = call(H, q, k, v, cu_q, cu_k, 1)
    H.hilo_sync_status()
    for i in range(n_q):
        back = n_q - 1 - i  # keys from the end that query i does not see
        row = got[2 + i].float()
        if back == 0:
            assert bool(row.isnan().all())
            continue
        want = base[2 + i].float().clone()
        for b, col, value in ((1, 70, math.nan), (37, 9, -math.inf), (64, 127, math.inf)):
            if b >= back:
                want[:, col] = value
        assert torch.equal(row.nan_to_num(7e4, 8e4, 9e4), want.nan_to_num(7e4, 8e4, 9e4)), (i, back)


@pytest.mark.parametrize("hd,heads,kv", [(128, 24, 4), (64, 32, 8)])
def test_rows_behind_a_long_cache(H, hd, heads, kv):
    """The last tile of a cache that keeps every SM loading: its rows behind the sequence are taken out after they
    have arrived, also where values come long after keys."""
    lk = [777, 20000, 64, 9001, 12345, 30001, 16000, 32700]
    q, k, v, cu_q, cu_k = make([1] * 8, lk, heads, kv, hd, "bf16", spare=200, seed=hd)
    k[sum(lk):], v[sum(lk):] = math.nan, math.nan
    ref = reference(q, k, v, cu_q, cu_k, 1)
    for _ in range(10):
        check(call(H, q, k, v, cu_q, cu_k, 1), ref, "bf16")
    # a last sequence of a single row of tiles too, at every remainder
    for n in (31997, 32001, 32100):
        cu = cu_k.clone()
        cu[-1] = cu[-2] + n
        k[int(cu[-1]):], v[int(cu[-1]):] = math.nan, math.nan
        got = call(H, q, k, v, cu_q, cu, 1)
        check(got[7:8], tuple(x[7:8] if hasattr(x, "shape") else x for x in reference(q[:8], k, v, cu_q, cu, 1)), "bf16")
        k.nan_to_num_(0.5), v.nan_to_num_(0.5)


def test_infinite_logits(H):
    """-inf logits weigh nothing, also where a query's first tile holds nothing else; all -inf gives NaN, as 0/0."""
    q, k, v, cu_q, cu_k = make([3, 40], [400, 300], 2, 1, 64, "bf16", seed=8)
    q[:, :, 0] = 1
    k[:200, :, 0] = -math.inf
    k[400:, :, 0] = -math.inf
    got = call(H, q, k, v, cu_q, cu_k, 0)
    cu2 = torch.tensor([200, 400], dtype=torch.int32, device="cuda")
    ref = reference(q[:3], k[:400], v[:400], cu_q[:2], cu2, 0)
    check(got[:3], ref, "bf16")
    assert bool(got[3:].isnan().all())


def test_calls_repeat_and_overlap(H):
    """The same bits again, on another stream, from a captured graph, and next to a call with a workspace of its own."""
    q, k, v, cu_q, cu_k = make([1, 1, 200], [3000, 900, 2500], 8, 2, 128, "bf16", seed=4)
    first = call(H, q, k, v, cu_q, cu_k)
    assert torch.equal(first, call(H, q, k, v, cu_q, cu_k))
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = []
    for _ in range(3):
        for s in (s1, s2):
            with torch.cuda.stream(s):
                outs.append(call(H, q, k, v, cu_q, cu_k))
    torch.cuda.synchronize()
    assert all(torch.equal(first, o) for o in outs)
    out = torch.zeros_like(q)
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    call(H, q, k, v, cu_q, cu_k, out=out, ws=ws)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(H, q, k, v, cu_q, cu_k, out=out, ws=ws)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, out)
    # the lengths are read at replay
    cu_q.copy_(torch.tensor([0, 1, 1, 150], dtype=torch.int32))
    cu_k.copy_(torch.tensor([0, 2000, 2000, 2900], dtype=torch.int32))
    out.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    check(out, reference(q, k, v, cu_q, cu_k, 1), "bf16")


def test_offsets_past_the_buffers_are_cut(H):
    """Offsets beyond the rows that the shape names (and falling ones) address nothing outside them."""
    q, k, v, cu_q, cu_k = make([100], [100], 2, 2, 64, "bf16", seed=6)
    store = torch.full((160, 2, 64), math.nan, dtype=q.dtype, device="cuda")
    cu_q = torch.tensor([-5, 90, 40, 150], dtype=torch.int32, device="cuda")
    cu_k = torch.tensor([0, 90, 95, 1 << 30], dtype=torch.int32, device="cuda")
    call(H, q, k, v, cu_q, cu_k, out=store[:100])
    H.hilo_sync_status()
    assert bool(store[100:].isnan().all())
    one = torch.tensor([0, 90], dtype=torch.int32, device="cuda")
    ref = reference(q[:90], k[:90], v[:90], one, one, 1)
    # (the third sequence, rows 40 to 99, overwrites the first one's later rows)
    check(store[:40], tuple(x[:40] if hasattr(x, "shape") else x for x in ref), "bf16")


def test_falling_offsets_that_name_rows_again_and_again(H):
    """More query tiles than rows and sequences can have: no row is written, and the next call is whole."""
    rows = 40000
    q = torch.randn(rows, 128, 64, device="cuda", dtype=torch.bfloat16)
    k = torch.randn(64, 1, 64, device="cuda", dtype=torch.bfloat16)
    cu_q = torch.tensor([0, rows] * 500, dtype=torch.int32, device="cuda")
    cu_k = torch.tensor([0, 64] * 500, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, math.nan)
    call(H, q, k, k, cu_q, cu_k, 0, out=out)
    H.hilo_sync_status()
    assert bool(out.isnan().all())
    one = [torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (200, 64)]
    check(call(H, q[:200], k, k, *one, 0), reference(q[:200], k, k, *one, 0), "bf16")


def test_no_keys_at_all(H):
    q, k, v, _, _ = make([4], [1], 2, 2, 64, "bf16")
    cu_q = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert bool((call(H, q, k[:0], v[:0], cu_q, zero, 0) == 0).all())
    assert bool(call(H, q, k, v, zero, zero, 0).isnan().all())


def single(hd, lk, low, seed, causal):
    """One query over lk keys in 2 key heads, the first `low` of them with logits of 200 below the others'."""
    q, k, v, cu_q, cu_k = make([1], [lk], 8, 2, hd, "bf16", seed=seed)
    q[:, :, 0], k[:, :, 0] = math.sqrt(hd), 0  # (the logit of channel 0 is k's)
    k[:low, :, 0] = -200
    return q, k, v, cu_q, cu_k


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("hd", [64, 128])
def test_seen_values_of_no_weight(H, hd, causal):
    """Infinities and NaNs that a query sees with a probability below the smallest fp32 number: 0 times them is NaN,
    whether the sequence is cut into pieces, is one job among many, or its steps follow one another."""
    lk, low, copies = 1300, 700, 200
    q, k, v, cu_q, cu_k = single(hd, lk, low, hd + causal, causal)
    clean = reference(q, k, v, cu_q, cu_k, causal)
    v[10, :, 5], v[300, :, 9], v[650, 1, 33] = math.nan, math.inf, -math.inf
    bad = torch.zeros(8, hd, dtype=torch.bool, device="cuda")
    bad[:, 5] = bad[:, 9] = bad[4:, 33] = True
    cut = call(H, q, k, v, cu_q, cu_k, causal)                      # 2 jobs on 152 CTAs: pieces
    many = [torch.arange(copies + 1, dtype=torch.int32, device="cuda") * n for n in (1, lk)]
    whole = call(H, *(x.repeat(copies, 1, 1) for x in (q, k, v)), *many, causal)  # 400 equal jobs: none is cut
    H.hilo_sync_status()
    for got in [cut[0], *whole]:
        assert torch.equal(~got.isfinite(), bad)
        fine = torch.where(bad, clean[0][0].to(got.dtype), got)[None]
        check(fine, clean, "bf16")


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("lq,lk,heads", [([300], [300], 2), ([90], [1400], 4), ([1], [500], 4), ([200, 130], [450, 130], 12)])
def test_infinities_and_nans_of_heads_of_64(H, dtype, causal, lq, lk, heads):
    """As test_infinities_and_nans_of_unseen_keys; without an order every query sees every key of its sequence."""
    q, k, v, cu_q, cu_k = make(lq, lk, heads, 2, 64, dtype, first=2, spare=6, seed=15)
    k[:2], v[:2], k[-6:], v[-6:] = math.nan, math.inf, math.nan, math.nan
    base = call(H, q, k, v, cu_q, cu_k, causal)
    sound = [x.clone() for x in (k, v)]
    for x in sound:
        x[:2], x[-6:] = 0, 0
    check(base, reference(q, *sound, cu_q, cu_k, causal), dtype)
    marks = ((0, 5, math.inf), (1, 40, math.nan), (37, 9, -math.inf), (64, 63, math.inf), (129, 20, math.nan))
    ends, q_ends = cu_k.tolist()[1:], cu_q.tolist()
    for end, n in zip(ends, lk):
        for back, col, value in marks:
            if back < n:
                v[end - 1 - back, :, col] = value
    got = call(H, q, k, v, cu_q, cu_k, causal)
    H.hilo_sync_status()
    for b, (n_q, n_k) in enumerate(zip(lq, lk)):
        for i in range(n_q):
            hidden = n_q - 1 - i if causal else 0  # keys from the end that query i does not see
            row, want = got[q_ends[b] + i].float(), base[q_ends[b] + i].float().clone()
            for back, col, value in marks:
                if hidden <= back < n_k:
                    want[:, col] = value
            assert torch.equal(row.nan_to_num(7e4, 8e4, 9e4), want.nan_to_num(7e4, 8e4, 9e4)), (b, i)


@pytest.mark.parametrize("lq,hd", [(1, 64), (1, 128), (200, 64), (200, 128)])
def test_small_probabilities_in_f16(H, lq, hd):
    """Many keys of 2^-26.5 of the largest probability each: below fp16's smallest number, but together all there is of the
    result. Probabilities are held against 2^7 or more for the largest, so a key is off by at most half of 2^-24 / 2^7."""
    lk = 512
    q, k, v, cu_q, cu_k = make([lq], [lk], 4, 2, hd, "f16")
    q[:], k[:], v[:] = 0, 0, 49152
    q[:, :, 0] = 1
    for top in (0, 128):  # the largest in both halves of the keys
        k[top, :, 0], v[top] = 18.375, 0
    o, mag, keys = reference(q, k, v, cu_q, cu_k, 0, scale=1.0)
    got = call(H, q, k, v, cu_q, cu_k, 0, scale=1.0).double()
    u = 2.0 ** -11
    tol = (u + 2.0 ** -13) * mag + u * o.abs() + keys * 2.0 ** -32 * 49152
    assert 0.1 < float(o.min()) and float((tol / o).max()) < 0.05
    assert bool(((got - o).abs() <= tol).all()), float(got.min())


def test_one_long_context_among_more_sequences_than_the_table_lists(H):
    """1100 single tokens, one of them over a long context: that one is cut into pieces as it is among 1000, and not the
    work of a single CTA. Right in either case, and of about the same time (a tenth more sequences; uncut the long one
    alone takes some ten times the call)."""
    def one(n, causal=1):
        lk = [1 + (37 * i) % 200 for i in range(n)]
        lk[n // 3] = 131072
        return make([1] * n, lk, 4, 1, 128, "bf16", seed=n)

    def time(args):
        ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
        out = torch.full(args[0].shape, math.nan, dtype=torch.bfloat16, device="cuda")
        best = math.inf
        for _ in range(5):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            call(H, *args, out=out, ws=ws)
            a.record()
            for _ in range(5):
                call(H, *args, out=out, ws=ws)
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b) / 5)
        H.hilo_sync_status()
        return best, out

    few, many = one(1000), one(1100)
    t_few, out = time(few)
    check(out, reference(*few, 1), "bf16")
    t_many, out = time(many)
    check(out, reference(*many, 1), "bf16")
    assert t_many < 3 * t_few, (t_few, t_many)


BEYOND = [
    # lq, lk, heads, kv heads, head_dim, causal, dtype: more than 1024 row jobs, some longer than a CTA's share
    ([1] * 1500, [90 + i % 300 for i in range(1499)] + [40000], 4, 2, 64, 1, "bf16"),
    ([1] * 2000, [60000] + [1 + i % 90 for i in range(1998)] + [30000], 3, 1, 128, 0, "f16"),
    ([1, 0] * 1200, [5 if i % 800 else 20000 for i in range(2400)], 2, 1, 128, 1, "bf16"),
    ([1200] * 9 + [200, 3], [1200] * 9 + [9000, 70000], 128, 1, 64, 1, "bf16"),   # few sequences of many tiles
    ([700] * 3 + [261], [90] * 3 + [50000], 128, 1, 64, 0, "f16"),                # a pair and a single at a sequence's end
    ([2] * 1100 + [64], [3] * 1100 + [30000], 4, 1, 64, 1, "bf16"),
]


@pytest.mark.parametrize("lq,lk,heads,kv,hd,causal,dtype", BEYOND)
def test_long_jobs_beyond_the_table(H, lq, lk, heads, kv, hd, causal, dtype):
    q, k, v, cu_q, cu_k = make(lq, lk, heads, kv, hd, dtype, first=3, spare=5, seed=len(lq) + sum(lk))
    got = call(H, q, k, v, cu_q, cu_k, causal)
    assert torch.equal(got.view(torch.int16), call(H, q, k, v, cu_q, cu_k, causal).view(torch.int16))
    H.hilo_sync_status()
    check(got, reference(q, k, v, cu_q, cu_k, causal), dtype)
