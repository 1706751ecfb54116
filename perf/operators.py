"""The conditioning and position operators of the block, as measurable cases.

Four operators, through the binding's public entry points where `own` is true
and in elementary torch operations where it is not:

  attn   hilo_attention: softmax attention of packed sequences with grouped
         heads, causal or not, whole prompts, chunks and single tokens
  rope   hilo_rope: rotary positions of several axes on the heads of rows
  norm   hilo_gate_norm: a branch's norm, gate and residual, and the next
         sub-layer's norm and modulation, over the text and image rows
  pos    hilo_row_positions: the positions of a split's packed rows

Values: queries, keys and values N(0,1) (queries doubled, as after a norm with
a learned gain), residual rows N(0,1) with a channel-dependent offset and gain,
branch rows N(0,1), modulation vectors N(0, 0.3^2), gates N(0, 0.5^2),
positions of a time x height x width grid with the half and quarter steps that
pooled rows have, labels random. All drawn on the GPU from the seed.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CODES = {"bf16": 0, "f32": 1, "f16": 2}  # HILO_BF16, HILO_F32, HILO_F16


# ----------------------------------------------------------------- cases ---


def _attn(name=None, **kw):
    """q, k: tokens of each sequence, new ones and those that they attend to. layout: q, k and v in the rows of
    one product ("fused"), in tensors of their own ("rows"), or k and v as a cache ordered by head ("heads")."""
    c = dict(op="attn", q="64", k="64", heads=8, kv_heads=8, hd=64, causal=1, dtype="bf16", layout="rows", spare=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def _rope(name=None, **kw):
    c = dict(op="rope", rows=1024, spare=0, heads=48, hd=128, dims="16,56,56", dtype="bf16", interleaved=1, per_axis=1,
             theta=10000.0, far=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def _norm(name=None, **kw):
    """parts: "in" (norm and modulation), "mid" (gate, residual, norm, modulation) or "out" (gate and residual)."""
    c = dict(op="norm", T=512, rows="1877", spare=0, d=3072, parts="mid", norm="layer", branch="none", u="f32", y="bf16",
             h="bf16", vec="bf16", resid=1.0, weights=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def _pos(name=None, **kw):
    c = dict(op="pos", B=1, H=64, W=64, d=512, T=512, levels=1, keep=0.3)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the next token of four short prompts: the smallest call, where latency counts
        _attn("attn_tokens_4", q="1,1,1,1", k="77,200,33,512", heads=8, kv_heads=2, hd=64, layout="heads", spare=64),
        # the prompts of a batch, packed, straight from the q|k|v product; one of them of a single token
        _attn("attn_prompts_ragged", q="512,77,1,333,200,1021", k="512,77,1,333,200,1021", heads=24, kv_heads=8, hd=128,
              layout="fused"),
        # one long document
        _attn("attn_prompt_8192", q="8192", k="8192", heads=32, kv_heads=8, hd=128),
        # images without an order between their tokens, one head of keys for each of queries
        _attn("attn_images_f16", q="2389,1111,4096", k="2389,1111,4096", heads=16, kv_heads=16, hd=64, causal=0, dtype="f16"),
        # the next token of sixteen requests whose contexts differ by four orders of magnitude
        _attn("attn_tokens_long", q=",".join("1" * 16),
              k="32768,8191,4096,1,2500,777,16000,64,12345,129,3333,9001,511,5000,1024,20000",
              heads=24, kv_heads=4, hd=128, layout="heads", spare=1000),
        # q and k heads of the main workload's compressed rows
        _rope("rope_rows_2389", rows=2389, heads=48, hd=128),
        # every row of a batch of four with its text, fp32, positions of a long video
        _rope("rope_far_f32", rows=18001, spare=200, heads=16, hd=64, dims="16,24,24", dtype="f32", interleaved=0, per_axis=0,
              theta=1000000.0, far=1),
        # the first norm of a block on a small grid
        _norm("norm_in_1024", T=64, rows="960", d=512, parts="in", u="bf16"),
        # between attention and MLP of the main workload
        _norm("norm_mid_2389"),
        # a batch of ragged images, norms on both sides of the branch
        _norm("norm_sandwich_b3", T=77, rows="3333,1021,4001", spare=300, d=1152, norm="rms", branch="rms", u="bf16",
              h="f16", vec="f32", resid=0.5, weights=1),
        # positions of one image's rows, and of a batch with two pooling levels
        _pos("pos_64"),
        _pos("pos_b4_128_two_level", B=4, H=128, W=128, levels=2, keep=0.2),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _draw_attn(rng):
    kv = rng.choice((1, 2, 4, 8))
    g = rng.choice((1, 1, 2, 3, 4, 6, 8))
    hd = rng.choice((64, 128))
    mode = rng.choice(("prompt", "prompt", "chunk", "token"))
    B = int(_log(rng, 1, 33))
    k = [int(_log(rng, 1, 16384 if mode == "token" else 6000)) for _ in range(B)]
    q = list(k)
    if mode == "token":
        q = [1] * B
    elif mode == "chunk":  # now and then longer than what it attends to: its first rows then see no key
        q = [int(_log(rng, 1, 1024)) for n in k]
        q = [min(a, n) if rng.random() < 0.8 else a for a, n in zip(q, k)]
    # no dearer than the longest listed one, in the padded plain form too
    while len(k) > 1 and len(k) * max(q) * max(k) * kv * g > 32 * 8192 * 8192:
        q.pop()
        k.pop()
    same = mode == "prompt"
    if rng.random() < 0.2:
        k.append(0)  # a sequence that is not there yet
        q.append(0 if same else rng.choice((0, 1, 3)))
    return _attn(q=",".join(map(str, q)), k=",".join(map(str, k)), heads=kv * g, kv_heads=kv, hd=hd,
                 causal=int(rng.random() < 0.8), dtype=rng.choice(("bf16", "bf16", "f16")),
                 layout=rng.choice(("fused", "rows") if same else ("rows", "heads")), spare=rng.choice((0, 0, 130)))


def draw(rng):
    op = rng.choice(("attn", "attn", "attn", "rope", "rope", "norm", "norm", "norm", "pos"))
    if op == "attn":
        return _draw_attn(rng)
    if op == "rope":
        hd, dims = rng.choice(((64, "16,24,24"), (64, "32,32"), (128, "16,56,56"), (128, "44,42,42"), (128, "64"),
                               (256, "64,96,96"), (80, "16,32,32"), (96, "24,24,24,24")))
        return _rope(rows=int(_log(rng, 1, 9000)), spare=rng.choice((0, 50)), heads=rng.choice((1, 3, 8, 16, 28, 48)), hd=hd,
                     dims=dims, dtype=rng.choice(("bf16", "bf16", "f16", "f32")),
                     interleaved=int(dims in ("44,42,42",) or rng.random() < 0.5), per_axis=rng.choice((0, 1)),
                     theta=rng.choice((256.0, 10000.0, 1000000.0)), far=rng.choice((0, 0, 1)))
    if op == "norm":
        B = rng.choice((1, 1, 2, 3, 5))
        parts = rng.choice(("in", "mid", "mid", "out"))
        return _norm(T=rng.choice((0, 64, 77, 200, 512)), rows=",".join(str(int(_log(rng, 1, 4096))) for _ in range(B)),
                     spare=rng.choice((0, 111)), d=8 * int(_log(rng, 8, 513)), parts=parts,
                     norm=rng.choice(("layer", "rms")), branch=rng.choice(("none", "layer", "rms")) if parts != "in" else "none",
                     u=rng.choice(("f32", "bf16")), y=rng.choice(("bf16", "f32")), h=rng.choice(("bf16", "f16", "f32")),
                     vec=rng.choice(("bf16", "f32")), resid=rng.choice((1.0, 1.0, 0.7071)), weights=rng.choice((0, 1)))
    levels = rng.choice((1, 2))
    return _pos(B=rng.choice((1, 2, 3, 4)), H=4 * int(_log(rng, 4, 33)), W=4 * int(_log(rng, 4, 33)), T=rng.choice((0, 77, 512)),
                levels=levels, keep=round(rng.uniform(0.0, 0.6), 3))


# ---------------------------------------------------------------- inputs ---


def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + salt)
    return g


def _ints(text):
    return [int(v) for v in text.split(",")]


def _offsets(lens):
    o = [0]
    for n in lens:
        o.append(o[-1] + n)
    return torch.tensor(o, dtype=torch.int32, device=DEV)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _prepare_attn(c, seed):
    g = _gen(seed, 1)
    lq, lk, hq, hk, hd, t = _ints(c["q"]), _ints(c["k"]), c["heads"], c["kv_heads"], c["hd"], TYPES[c["dtype"]]
    nq, nk = sum(lq) + c["spare"], sum(lk) + c["spare"]
    q = (2 * _randn(g, nq, hq, hd)).to(t)
    k, v = _randn(g, nk, hk, hd).to(t), _randn(g, nk, hk, hd).to(t)
    k[sum(lk):], v[sum(lk):] = float("nan"), float("nan")  # rows behind the last sequence: whatever was there
    if c["layout"] == "fused":
        rows = torch.cat([x.reshape(nq, -1) for x in (q, k, v)], 1)
        q, k, v = (x.unflatten(1, (-1, hd)) for x in rows.split([hq * hd, hk * hd, hk * hd], 1))
    elif c["layout"] == "heads":
        k, v = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (k, v))
    s = dict(c, qs=q, ks=k, vs=v, cu_q=_offsets(lq), cu_k=_offsets(lk), lq=max(lq), lk=max(lk),
             out=torch.zeros(nq, hq, hd, dtype=t, device=DEV))
    if own:
        from paper_2606_13898_gb300 import hilo as H
        s["shape"] = H.AttnShape(B=len(lq), heads=hq, kv_heads=hk, head_dim=hd, rows_q=nq, rows_k=nk, causal=c["causal"],
                                 dtype=CODES[c["dtype"]], q_row=q.stride(0), q_head=q.stride(1), k_row=k.stride(0),
                                 k_head=k.stride(1), v_row=v.stride(0), v_head=v.stride(1))
        s["ws_bytes"] = H.hilo_attention_workspace_bytes(s["shape"])
        s["ws"] = torch.empty(s["ws_bytes"], dtype=torch.uint8, device=DEV)
    return s


def _prepare_rope(c, seed):
    g = _gen(seed, 2)
    n, cap, axes = c["rows"], c["rows"] + c["spare"], len(_ints(c["dims"]))
    x = _randn(g, cap, c["heads"], c["hd"]).to(TYPES[c["dtype"]])
    side = max(2, int(math.sqrt(n)))
    grid = torch.randint(0, 4 * side, (cap, axes), generator=g, device=DEV).float() / 4
    if c["far"]:
        grid[:, 0] += 30000.0 + 7.0 * torch.arange(cap, device=DEV)
    s = dict(c, x=x, pos=grid, n_rows=torch.tensor([n], dtype=torch.int32, device=DEV), out=torch.zeros_like(x),
             pairs=_pairs(c))
    if own:
        from paper_2606_13898_gb300 import hilo as H
        s["shape"] = H.RopeShape(rows=cap, heads=c["heads"], head_dim=c["hd"], dtype=CODES[c["dtype"]],
                                 axis_dims=tuple(_ints(c["dims"])), theta=c["theta"], interleaved=c["interleaved"],
                                 per_axis=c["per_axis"])
    return s


def _prepare_norm(c, seed):
    g = _gen(seed, 3)
    rows, d, T = _ints(c["rows"]), c["d"], c["T"]
    B, cap = len(rows), sum(rows) + c["spare"]
    R = B * T + cap
    u = _randn(g, R, d) * (0.5 + torch.rand(d, generator=g, device=DEV)) + 0.3 * _randn(g, d)
    vt = TYPES[c["vec"]]
    # the vectors of one product of the time embedding: shift | scale | gate of image b in row b
    mod = [(0.3 * _randn(g, B, 3 * d)).to(vt) for _ in range(2)]
    for m in mod:
        m[:, 2 * d:] *= 5 / 3
    w = [(1 + 0.1 * _randn(g, 3, d)).to(vt) for _ in range(2)]
    s = dict(c, u_rows=u.to(TYPES[c["u"]]), y_rows=_randn(g, R, d).to(TYPES[c["y"]]), mod=mod, w=w, cu=_offsets(rows), n=B,
             u_out=torch.zeros(R, d, dtype=TYPES[c["u"]], device=DEV), h_out=torch.zeros(R, d, dtype=TYPES[c["h"]], device=DEV))
    if own:
        from paper_2606_13898_gb300 import hilo as H
        kinds = {"none": H.HILO_NORM_NONE, "layer": H.HILO_NORM_LAYER, "rms": H.HILO_NORM_RMS}
        last = c["parts"] == "out"
        s["shape"] = H.NormShape(B=B, T=T, cap=cap, d=d, norm=kinds["none" if last else c["norm"]], norm_branch=kinds[c["branch"]],
                                 eps=1e-6, resid_scale=c["resid"], u_dtype=CODES[c["u"]], y_dtype=CODES[c["y"]],
                                 u_out_dtype=CODES[c["u"]], h_dtype=CODES[c["h"]], vec_dtype=CODES[c["vec"]], vec_row=3 * d)
        s["vectors"] = [H.NormVectors(gate=None if c["parts"] == "in" else m[:, 2 * d:], scale=None if last else m[:, d:2 * d],
                                      shift=None if last else m[:, :d],
                                      w_branch=x[0] if c["weights"] and c["branch"] != "none" else None,
                                      w_norm=x[1] if c["weights"] and not last else None,
                                      b_norm=x[2] if c["weights"] and not last else None) for m, x in zip(mod, w)]
    return s


def _prepare_pos(c, seed):
    g = _gen(seed, 4)
    B, H_, W_, levels = c["B"], c["H"], c["W"], c["levels"]
    kept = torch.rand(B, H_, W_, generator=g, device=DEV) < c["keep"]
    fine = torch.rand(B, H_, W_, generator=g, device=DEV) < (0.5 if levels == 2 else 1.1)
    labels = torch.where(kept, 0, torch.where(fine, 1, 2)).to(torch.uint8)

    def windows(label, n):
        has = (labels == label).view(B, H_ // n, n, W_ // n, n).any(4).any(2)
        return has.view(B, -1)

    parts = [(labels == 0).view(B, -1), windows(1, 2), windows(2, 4)]
    counts = torch.stack([p.sum(1) for p in parts], 1).to(torch.int32)
    per = [[p[b].nonzero().view(-1) for p in parts] for b in range(B)]
    src = torch.cat([x for image in per for x in image]).to(torch.int32)
    cap = B * H_ * W_
    row_src = torch.zeros(cap, dtype=torch.int32, device=DEV)
    row_src[:src.numel()] = src
    cu = torch.cat([torch.zeros(1, dtype=torch.int32, device=DEV), counts.sum(1).cumsum(0).to(torch.int32)])
    s = dict(c, labels=labels.view(-1), row_src=row_src, counts=counts, cu=cu, cap=cap,
             out=torch.zeros(B * c["T"] + cap, 3, dtype=torch.float32, device=DEV))
    if own:
        from paper_2606_13898_gb300 import hilo as H
        s["shape"] = H.Shape(B=B, H=H_, W=W_, d=c["d"], T=c["T"], heads=c["d"] // 64, levels=levels)
        s["split"] = H.SplitBuffers(s["labels"], row_src, counts.view(-1), cu, torch.zeros(cap, dtype=torch.int32, device=DEV))
        s["origin"] = H.RowPositions(t_img=1.0, h0=-0.5 * H_, w0=-0.5 * W_, txt0=0.5 * H_, txt_step=1.0)
    return s


def prepare(case, seed):
    return {"attn": _prepare_attn, "rope": _prepare_rope, "norm": _prepare_norm, "pos": _prepare_pos}[case["op"]](case, seed)


# ------------------------------------------------------------------ plain ---


def _padded(cu, most):
    """Row numbers [B, most] of each sequence, and which of them it has."""
    at = torch.arange(most, device=DEV)
    n = (cu[1:] - cu[:-1]).long()
    there = at < n[:, None]
    return torch.where(there, cu[:-1, None].long() + at, 0), there, n


def _plain_attn(s):
    B, hq, hk, hd = s["cu_q"].numel() - 1, s["heads"], s["kv_heads"], s["hd"]
    at_q, in_q, nq = _padded(s["cu_q"], s["lq"])
    at_k, in_k, nk = _padded(s["cu_k"], s["lk"])
    g, lq, lk = hq // hk, s["lq"], s["lk"]
    q = s["qs"][at_q].float().view(B, lq, hk, g, hd).permute(0, 2, 3, 1, 4).reshape(B, hk, g * lq, hd)
    k = s["ks"][at_k].float().permute(0, 2, 3, 1)
    v = s["vs"][at_k].float().permute(0, 2, 1, 3)
    seen = in_k[:, None, :] & in_q[:, :, None]
    if s["causal"]:
        i, j = torch.arange(lq, device=DEV), torch.arange(lk, device=DEV)
        seen = seen & (j <= (i[:, None] + (nk - nq)[:, None, None]))
    x = torch.matmul(q, k).mul_(1 / math.sqrt(hd)).view(B, hk, g, lq, lk)
    x.masked_fill_(~seen[:, None, None], float("-inf"))
    top = x.amax(-1, keepdim=True)
    x.sub_(torch.where(torch.isinf(top), 0.0, top)).exp_()
    total = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, hk, g * lq, lk), v).view(B, hk, g, lq, hd) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, lq, hq, hd)
    r, cu = torch.arange(s["qs"].shape[0], device=DEV), s["cu_q"].long()
    b = torch.searchsorted(cu[1:], r, right=True).clamp(max=B - 1)
    i = (r - cu[b]).clamp(max=lq - 1)
    return torch.where((r < cu[-1])[:, None, None], o[b, i], 0.0).to(s["out"].dtype)


def _pairs(c):
    """Axis and frequency of each rotated pair, and the channels of its two members."""
    dims = _ints(c["dims"])
    D = sum(dims)
    axis = [a for a, n in enumerate(dims) for _ in range(n // 2)]
    part = [i / n for n in dims for i in range(0, n, 2)] if c["per_axis"] else [i / D for i in range(0, D, 2)]
    first = [2 * i for i in range(D // 2)] if c["interleaved"] else list(range(D // 2))
    step = 1 if c["interleaved"] else D // 2
    freq = torch.tensor([c["theta"] ** -p for p in part], dtype=torch.float64, device=DEV)
    return [torch.tensor(axis, device=DEV), freq] + [torch.tensor([i + k for i in first], device=DEV) for k in (0, step)]


def _plain_rope(s):
    (axis, freq, a, b), n = s["pairs"], s["rows"]
    angle = s["pos"][:n, axis].double() * freq
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    x = s["x"][:n].float()
    y = x.clone()
    y[:, :, a] = x[:, :, a] * cos - x[:, :, b] * sin
    y[:, :, b] = x[:, :, a] * sin + x[:, :, b] * cos
    out = torch.zeros_like(s["x"])
    out[:n] = y.to(out.dtype)
    return out


def _image_of(s):
    """The rows that there are, and the image and stream of each."""
    B, T = s["n"], s["T"]
    R = s["u_rows"].shape[0]
    r = torch.arange(R, device=DEV)
    img = r - B * T
    b = torch.where(img < 0, r // max(T, 1), torch.searchsorted(s["cu"].long(), img.clamp(min=0), right=True) - 1)
    there = img < s["cu"][-1]
    return b.clamp(max=B - 1), img < 0, there


def _plain_norm(s):
    d, eps = s["d"], 1e-6
    b, is_txt, there = _image_of(s)
    pick = lambda v: torch.where(is_txt[:, None], v[0].float()[b], v[1].float()[b])  # noqa: E731
    each = lambda i: torch.where(is_txt[:, None], s["w"][0][i].float(), s["w"][1][i].float())  # noqa: E731

    def norm(x, kind):
        if kind == "none":
            return x
        if kind == "layer":
            x = x - x.mean(-1, keepdim=True)
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps)

    shift, scale, gate = (pick([m[:, i * d:(i + 1) * d] for m in s["mod"]]) for i in range(3))
    u = s["u_rows"].float()
    outs = {}
    if s["parts"] != "in":
        z = norm(s["y_rows"].float(), s["branch"])
        if s["weights"] and s["branch"] != "none":
            z = z * each(0)
        u = s["resid"] * u + gate * z
        outs["u"] = torch.where(there[:, None], u, 0.0).to(s["u_out"].dtype)
    if s["parts"] != "out":
        h = norm(u, s["norm"])
        if s["weights"]:
            h = h * each(1) + each(2)
        outs["h"] = torch.where(there[:, None], h * (1 + scale) + shift, 0.0).to(s["h_out"].dtype)
    return outs


def _plain_pos(s):
    B, H_, W_, T = s["B"], s["H"], s["W"], s["T"]
    out = torch.zeros_like(s["out"])
    txt = 0.5 * H_ + torch.arange(T, device=DEV).float()
    out[:B * T] = txt.repeat(B)[:, None]
    lab = s["labels"].view(B, H_, W_)
    p = torch.arange(H_, device=DEV).float()[:, None].expand(H_, W_)
    q = torch.arange(W_, device=DEV).float()[None, :].expand(H_, W_)
    r, cu = torch.arange(s["cap"], device=DEV), s["cu"].long()
    b = torch.searchsorted(cu[1:], r, right=True).clamp(max=B - 1)
    local = r - cu[b]
    n = s["counts"].long()
    level = (local >= n[b, 0]).long() + (local >= n[b, 0] + n[b, 1]).long()
    src = s["row_src"].long()
    at = torch.zeros(s["cap"], 2, device=DEV)

    def window(label, k):
        m = (lab == label).view(B, H_ // k, k, W_ // k, k).float()
        count = m.sum((2, 4)).view(B, -1)
        mean = lambda v: (m * v.view(H_ // k, k, W_ // k, k)).sum((2, 4)).view(B, -1) / count  # noqa: E731
        return torch.stack([mean(p.contiguous()), mean(q.contiguous())], -1)

    kept = torch.stack([p.reshape(-1), q.reshape(-1)], -1)
    two, four = window(1, 2), window(2, 4)
    for_level = lambda k: torch.where(level == k, src, 0)  # noqa: E731
    at = torch.where((level == 0)[:, None], kept[for_level(0)], at)
    at = torch.where((level == 1)[:, None], two[b, for_level(1)], at)
    at = torch.where((level == 2)[:, None], four[b, for_level(2)], at)
    at = torch.cat([torch.ones_like(at[:, :1]), at[:, :1] - 0.5 * H_, at[:, 1:] - 0.5 * W_], 1)
    out[B * T:] = torch.where((r < cu[-1])[:, None], at, 0.0)
    return out


# --------------------------------------------------------------- one pass ---


def run(s):
    if not own:
        return {"attn": _plain_attn, "rope": _plain_rope, "norm": _plain_norm, "pos": _plain_pos}[s["op"]](s)
    from paper_2606_13898_gb300 import hilo as H
    if s["op"] == "attn":
        H.hilo_attention(s["shape"], s["cu_q"], s["cu_k"], s["qs"], s["ks"], s["vs"], s["out"], s["ws"], s["ws_bytes"])
        return s["out"]
    if s["op"] == "rope":
        H.hilo_rope(s["shape"], s["x"], s["pos"], s["n_rows"], s["out"])
        return s["out"]
    if s["op"] == "norm":
        first, last = s["parts"] == "in", s["parts"] == "out"
        text = s["n"] * s["T"]
        H.hilo_gate_norm(s["shape"], s["vectors"][0], s["vectors"][1], s["cu"], s["u_rows"], s["u_rows"][text:],
                         None if first else s["y_rows"], None if first else s["u_out"], None if last else s["h_out"], None)
        return {k: v for k, v in (("u", None if first else s["u_out"]), ("h", None if last else s["h_out"])) if v is not None}
    H.hilo_row_positions(s["shape"], s["split"], s["origin"], s["out"], s["cap"])
    return s["out"]


def _seen(lq, lk, causal):
    """Pairs of a query and a key that it sees."""
    if not causal:
        return lq * lk
    n = min(lq, lk)  # the last n queries see lk - n + 1 .. lk keys
    return n * (lk - n) + n * (n + 1) // 2


def work(c):
    size = {"bf16": 2, "f16": 2, "f32": 4}
    if c["op"] == "attn":
        lq, lk = _ints(c["q"]), _ints(c["k"])
        rows = 2 * sum(lq) * c["heads"] + 2 * sum(lk) * c["kv_heads"]
        seen = sum(_seen(a, b, c["causal"]) for a, b in zip(lq, lk))
        return {"bytes": rows * c["hd"] * 2, "flops": 4 * c["hd"] * c["heads"] * seen}
    if c["op"] == "rope":
        n = c["rows"]
        return {"bytes": 2 * n * c["heads"] * c["hd"] * size[c["dtype"]] + 4 * n * len(_ints(c["dims"])),
                "flops": 3 * n * c["heads"] * sum(_ints(c["dims"]))}
    if c["op"] == "norm":
        rows = _ints(c["rows"])
        n = len(rows) * c["T"] + sum(rows)
        first, last = c["parts"] == "in", c["parts"] == "out"
        each = size[c["u"]] + (0 if first else size[c["u"]] + size[c["y"]]) + (0 if last else size[c["h"]])
        vectors = (2 if first else 1 if last else 3) * (2 if c["T"] else 1) * len(rows) * size[c["vec"]]
        return {"bytes": n * c["d"] * each + vectors * c["d"], "flops": 12 * n * c["d"]}
    n = c["B"] * c["H"] * c["W"]
    rows = n * (c["keep"] + (1 - c["keep"]) / 3) + c["B"] * c["T"]
    return {"bytes": n + 16 * rows, "flops": 4 * n}


# ------------------------------------------------------------------ exact ---


def _exact_attn(s):
    q, k, v = s["qs"].double(), s["ks"].double(), s["vs"].double()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    cq, ck, g = s["cu_q"].tolist(), s["cu_k"].tolist(), s["heads"] // s["kv_heads"]
    for i in range(len(cq) - 1):
        q0, q1, k0, k1 = cq[i], cq[i + 1], ck[i], ck[i + 1]
        if q1 == q0 or k1 == k0:
            continue
        last = torch.arange(q1 - q0, device=DEV) + (k1 - k0) - (q1 - q0) if s["causal"] else \
            torch.full((q1 - q0,), k1 - k0 - 1, device=DEV)
        hidden = torch.arange(k1 - k0, device=DEV) > last[:, None]
        for h in range(s["heads"]):
            logit = q[q0:q1, h] @ k[k0:k1, h // g].T / math.sqrt(s["hd"])
            logit[hidden] = -math.inf
            w = torch.exp(logit - logit.amax(1, keepdim=True).clamp(min=-1e300))
            out[q0:q1, h] = (w @ v[k0:k1, h // g]) / w.sum(1, keepdim=True).clamp(min=1e-300)
    return out


def _exact_rope(s):
    dims, n = _ints(s["dims"]), s["rows"]
    D = sum(dims)
    x = s["x"][:n].double()
    out = torch.zeros(s["x"].shape, dtype=torch.float64, device=DEV)
    out[:n] = x
    i = 0
    for a, dim in enumerate(dims):
        for e in range(dim // 2):
            f = s["theta"] ** (-2.0 * e / dim) if s["per_axis"] else s["theta"] ** (-2.0 * i / D)
            z = torch.polar(torch.ones(n, dtype=torch.float64, device=DEV), s["pos"][:n, a].double() * f)[:, None]
            lo, hi = (2 * i, 2 * i + 1) if s["interleaved"] else (i, i + D // 2)
            r = torch.complex(x[..., lo], x[..., hi]) * z
            out[:n, :, lo], out[:n, :, hi] = r.real, r.imag
            i += 1
    return out


def _exact_norm(s):
    d, T, B = s["d"], s["T"], s["n"]
    R, cu = s["u_rows"].shape[0], s["cu"].tolist()
    res = {}
    if s["parts"] != "in":
        res["u"] = torch.zeros(R, d, dtype=torch.float64, device=DEV)
    if s["parts"] != "out":
        res["h"] = torch.zeros(R, d, dtype=torch.float64, device=DEV)

    def scaled(x, kind):
        if kind == "none":
            return x
        mean = x.mean(1, keepdim=True) if kind == "layer" else 0.0
        return (x - mean) / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + 1e-6)

    for stream in range(2):
        w = s["w"][stream].double()
        for b in range(B):
            lo, hi = (b * T, b * T + T) if stream == 0 else (B * T + cu[b], B * T + cu[b + 1])
            shift, scale, gate = s["mod"][stream][b].double().split(d)
            u = s["u_rows"][lo:hi].double()
            if s["parts"] != "in":
                z = scaled(s["y_rows"][lo:hi].double(), s["branch"])
                if s["weights"] and s["branch"] != "none":
                    z = z * w[0]
                u = s["resid"] * u + gate * z
                res["u"][lo:hi] = u
            if s["parts"] != "out":
                h = scaled(u, s["norm"])
                if s["weights"]:
                    h = h * w[1] + w[2]
                res["h"][lo:hi] = h * (1 + scale) + shift
    return res


def _exact_pos(s):
    B, H_, W_, T = s["B"], s["H"], s["W"], s["T"]
    lab, src, n = s["labels"].view(B, H_, W_).cpu(), s["row_src"].tolist(), s["counts"].tolist()
    out = torch.zeros(s["out"].shape, dtype=torch.float64)
    for r in range(B * T):
        out[r] = 0.5 * H_ + r % T
    r = 0
    for b in range(B):
        image = lab[b].tolist()
        for label, side in ((0, 1), (1, 2), (2, 4)):
            for _ in range(n[b][label]):
                top, left = side * (src[r] // (W_ // side)), side * (src[r] % (W_ // side))
                at = [(p, q) for p in range(top, top + side) for q in range(left, left + side) if image[p][q] == label]
                out[B * T + r, 0] = 1.0
                out[B * T + r, 1] = sum(p for p, _ in at) / len(at) - 0.5 * H_
                out[B * T + r, 2] = sum(q for _, q in at) / len(at) - 0.5 * W_
                r += 1
    return out.to(DEV)


def exact(case, seed):
    s = prepare(case, seed)
    return {"attn": _exact_attn, "rope": _exact_rope, "norm": _exact_norm, "pos": _exact_pos}[case["op"]](s)
