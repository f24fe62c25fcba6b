"""Attention between all tokens of an image, as the point decoder's blocks and the last, shortest stages have it, and the rotary
positions of its queries and keys, as a program that uses this library has them done.

A case is a dict of plain values.  `op` names the call or calls of one pass:

  rotary_fwd   queries [B,N,H,d] and, with Hk > 0, keys [B,N,Hk,d] rotated by the tokens' positions: the pair c of a head's channels turns
               by the angle sum_a coords[b,n,a] freq[c,a] (2-D token coordinates, or time, height and width of a video's tokens)
  rotary_bwd   the gradients of both, and with `dcoords` those of the positions (the decoder's are learned)
  attn_fwd     out = softmax(s) v and lse, s = scale <q, k>, with `cap` cap tanh(s / cap), with `distance` less slope[h] |x_i - y_j|;
               with `docs` several images' tokens lie in one row and a token sees those of its own image only; Hk key heads serve H
               query heads
  attn_train   the same and its gradients dq, dk, dv (and dslope)

Where `own` is false `run` computes the operators with elementary torch operations in 32 bits, angles in 64.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
FRAME = 1024.0  # pixels


# ---------------------------------------------------------------------------------------------------------- the cases

def _rotary(name, op, dtype, B, N, H, Hk, d, axes=2, layout="pairs", dcoords=False, far=0.0):
    c = {"op": op, "dtype": dtype, "B": B, "N": N, "H": H, "Hk": Hk, "d": d, "axes": axes, "layout": layout, "dcoords": dcoords, "far": far}
    if name:
        c["name"] = name
    return c


def _attn(name, op, dtype, B, Nq, Nk, H, Hk, d, cap=0.0, distance=False, docs=0):
    """docs: images packed into each row (their lengths come with the inputs), the row's last 1/64 is padding; 0: no such mask."""
    c = {"op": op, "dtype": dtype, "B": B, "Nq": Nq, "Nk": Nk, "H": H, "Hk": Hk, "d": d, "cap": cap, "distance": distance, "docs": docs}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one image of 256 tokens in full precision: latency counts
        _rotary("rotary_tiny", "rotary_fwd", "f32", 1, 256, 2, 2, 32),
        # fine-tuning on 1024-px images, first stage: queries and keys of 8 images of 16384 tokens
        _rotary("rotary_finetune", "rotary_fwd", "bf16", 8, 16384, 2, 2, 32),
        # clips of a video: time, height and width; fewer key heads; channels paired across the halves of a head; odd token count
        _rotary("rotary_video", "rotary_fwd", "bf16", 4, 6271, 12, 4, 64, axes=3, layout="halves"),
        # training of the point decoder: 48 images of 2048 queries whose positions are learned
        _rotary("rotary_bwd_decoder", "rotary_bwd", "bf16", 48, 2048, 6, 0, 64, dcoords=True),
        # whatever sizes a head has, in full precision, on a crop of a mosaic whose coordinates run to millions of pixels
        _rotary("rotary_bwd_ragged", "rotary_bwd", "f32", 3, 4001, 3, 1, 24, far=2.0e6, dcoords=True),
        # one image of 256 tokens in full precision, scores falling with the distance
        _attn("attn_tiny", "attn_fwd", "f32", 1, 256, 256, 2, 2, 32, distance=True),
        # the decoder's self-attention at inference: 8 images of 4096 queries, six heads
        _attn("attn_decoder", "attn_fwd", "bf16", 8, 4096, 4096, 6, 6, 64),
        # a single query against every token of each of four images, four query heads to a key head
        _attn("attn_one_query", "attn_fwd", "bf16", 4, 1, 16384, 12, 3, 64, distance=True),
        # what masks leave of images, packed into rows without padding each to the longest; capped scores
        _attn("attn_packed", "attn_fwd", "bf16", 2, 8001, 8001, 4, 4, 32, cap=30.0, docs=11),
        # training of a merged stage with attention between all its tokens: 16 images of 1024 tokens, distances
        _attn("attn_train_merged", "attn_train", "bf16", 16, 1024, 1024, 8, 8, 32, distance=True),
        # the largest: training of a wide last stage
        _attn("attn_train_wide", "attn_train", "bf16", 8, 4096, 4096, 6, 6, 128),
        # the decoder's queries against what a mask leaves, full precision, sizes that nothing divides, all terms at once
        _attn("attn_train_ragged", "attn_train", "f32", 2, 1003, 777, 6, 2, 40, cap=20.0, distance=True, docs=3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary_fwd", "rotary_bwd", "attn_fwd", "attn_fwd", "attn_fwd", "attn_train", "attn_train", "attn_train"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op.startswith("rotary"):
        axes = rng.randint(1, 3)
        Hk = rng.choice([0, 1, 2, 4])
        H = rng.randint(1, 3) * max(Hk, 1)
        d = rng.choice([16, 32, 64, 128, 2 * rng.randint(2, 64)])
        N = _log(rng, 1, 16384)
        B = max(1, min(_log(rng, 1, 64), int(5e7 / (N * (H + Hk) * d))))
        return _rotary(None, op, dtype, B, N, H, Hk, d, axes, rng.choice(["pairs", "halves"]), op == "rotary_bwd" and rng.random() < 0.5,
                       rng.choice([0.0, 0.0, 1.0e4, 2.0e6]))
    Hk = rng.choice([1, 2, 3, 4, 6, 8])
    H = Hk * rng.choice([1, 1, 2, 3, 4])
    d = rng.choice([16, 32, 32, 64, 64, 128, 8 * rng.randint(1, 16)])
    docs = rng.choice([0, 0, 0, 1, rng.randint(2, 40)])
    Nk = max(_log(rng, 1, 16384), 2 * docs)
    Nq = rng.choice([Nk, Nk, max(_log(rng, 1, 4096), 2 * docs)])
    # a fraction of the largest listed case's pairs of tokens
    most = 1.5e8 if dtype == "bf16" else 3e7
    Nq = max(1, min(Nq, int(most / (Nk * H))))
    B = max(1, min(_log(rng, 1, 64), int(most / (Nk * Nq * H))))
    return _attn(None, op, dtype, B, Nq, Nk, H, Hk, d, rng.choice([0.0, 0.0, rng.uniform(5.0, 50.0)]), rng.random() < 0.4, min(docs, Nq // 2))


# --------------------------------------------------------------------------------------------------------- their inputs

def _images(g, B, N, docs):
    """Image of each of a row's tokens, in order, -1 in the padding at its end; images of N / docs tokens, more or less."""
    last = N - N // 64
    cuts = ((torch.arange(docs, device=DEV) + torch.rand(B, docs, generator=g, device=DEV)) * (last / docs)).long()
    cuts[:, 0] = 0
    place = torch.arange(N, device=DEV)
    ids = (place[None, :, None] >= cuts[:, None, :]).sum(dim=2) - 1
    return torch.where(place < last, ids, torch.full_like(ids, -1)).to(torch.int32)


def _inputs(case, seed):
    """The tensors that the call reads, from the seed alone."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t = TYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=g, device=DEV) * std).to(t)

    def places(B, N, axes=2):
        return torch.rand(B, N, axes, generator=g, device=DEV) * FRAME

    B, H, Hk, d = (case[n] for n in ("B", "H", "Hk", "d"))
    s = {}
    if case["op"].startswith("rotary"):
        N, axes = case["N"], case["axes"]
        s["coords"] = places(B, N, axes) + case["far"]
        # the axes take turns at the pairs of channels; wavelengths from two patches of 8 pixels to two frames
        c = torch.arange(d // 2, device=DEV)
        rate = math.pi / 8 * 128.0 ** (-(c // axes).double() / max(-(-(d // 2) // axes), 1))
        s["freq"] = torch.where(c[:, None] % axes == torch.arange(axes, device=DEV), rate[:, None], 0.0).float().contiguous()
        if case["op"] == "rotary_fwd":
            s["q"] = normal(B, N, H, d)
            s["k"] = normal(B, N, Hk, d) if Hk else None
        else:
            s["dq_out"] = normal(B, N, H, d)
            s["dk_out"] = normal(B, N, Hk, d) if Hk else None
            # what the forward pass returned (needed for the positions' gradients)
            s["q_out"] = normal(B, N, H, d) if case["dcoords"] else None
            s["k_out"] = normal(B, N, Hk, d) if case["dcoords"] and Hk else None
        return s
    Nq, Nk = case["Nq"], case["Nk"]
    s["q"], s["k"], s["v"] = normal(B, Nq, H, d), normal(B, Nk, Hk, d), normal(B, Nk, Hk, d)
    s["scale"] = d ** -0.5
    s["q_xy"] = s["k_xy"] = s["slope"] = s["q_doc"] = s["k_doc"] = None
    if case["distance"]:
        s["k_xy"] = places(B, Nk)
        s["q_xy"] = s["k_xy"] if Nq == Nk else places(B, Nq)
        # a score falls by one within 16 pixels in the narrowest head, within 256 in the widest
        s["slope"] = torch.logspace(-4, -8, H, base=2.0, device=DEV) * (torch.rand(H, generator=g, device=DEV) * 0.5 + 0.75)
    if case["docs"]:
        s["k_doc"] = _images(g, B, Nk, case["docs"])
        s["q_doc"] = s["k_doc"] if Nq == Nk else _images(g, B, Nq, case["docs"])
    if case["op"] == "attn_train":
        s["dout"] = normal(B, Nq, H, d)
    return s


def prepare(case, seed):
    s = dict(case)
    s.update(_inputs(case, seed))
    return s


# -------------------------------------------------------------------------------------------------- one pass, both ways

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2602_16249_amd as aff
    if s["op"] == "rotary_fwd":
        q, k = aff.affmae_rotary_fwd(s["q"], s["coords"], s["freq"], k=s["k"], layout=s["layout"])
        return {"q": q, "k": k} if k is not None else {"q": q}
    if s["op"] == "rotary_bwd":
        return aff.affmae_rotary_bwd(s["dq_out"], s["coords"], s["freq"], dk_out=s["dk_out"], layout=s["layout"], q_out=s["q_out"],
                                     k_out=s["k_out"], want_dcoords=s["dcoords"])
    terms = dict(cap=s["cap"], q_xy=s["q_xy"], k_xy=s["k_xy"], slope=s["slope"], q_doc=s["q_doc"], k_doc=s["k_doc"])
    out, lse = aff.affmae_attn_fwd(s["q"], s["k"], s["v"], s["scale"], **terms)
    r = {"out": out, "lse": lse}
    if s["op"] == "attn_train":
        r.update(aff.affmae_attn_bwd(s["q"], s["k"], s["v"], out, lse, s["dout"], s["scale"], **terms))
    return r


def _turned(x, cos, sin, layout):
    """The pairs of x [B,N,H,d] turned by angles with these [B,N,1,d/2] cosines and sines."""
    if layout == "pairs":
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    a, b = x.chunk(2, dim=-1)
    return torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)


def _spin(out, dout, layout):
    """What a pair's angle does to <dout, out>, summed over heads: [B,N,d/2]."""
    if layout == "pairs":
        return (out[..., 0::2] * dout[..., 1::2] - out[..., 1::2] * dout[..., 0::2]).sum(dim=2)
    half = out.shape[-1] // 2
    return (out[..., :half] * dout[..., half:] - out[..., half:] * dout[..., :half]).sum(dim=2)


def _run_plain_rotary(s):
    t, layout = TYPES[s["dtype"]], s["layout"]
    angle = (s["coords"].double()[:, :, None, :] * s["freq"].double()).sum(dim=-1)[:, :, None, :]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    if s["op"] == "rotary_fwd":
        r = {"q": _turned(s["q"].float(), cos, sin, layout).to(t)}
        if s["k"] is not None:
            r["k"] = _turned(s["k"].float(), cos, sin, layout).to(t)
        return r
    g = {"dq": _turned(s["dq_out"].float(), cos, -sin, layout).to(t)}
    if s["dk_out"] is not None:
        g["dk"] = _turned(s["dk_out"].float(), cos, -sin, layout).to(t)
    if s["dcoords"]:
        spin = _spin(s["q_out"].float(), s["dq_out"].float(), layout)
        if s["dk_out"] is not None:
            spin = spin + _spin(s["k_out"].float(), s["dk_out"].float(), layout)
        g["dcoords"] = (spin[..., None] * s["freq"]).sum(dim=2)
    return g


def _heads_first(x, heads):
    """[B,N,Hk,d] as [B,heads,N,d] in 32 bits, each of the Hk heads for heads / Hk of them."""
    return x.float().repeat_interleave(heads // x.shape[2], dim=2).permute(0, 2, 1, 3).contiguous()


def _shared(x, Hk, t):
    """Gradients [B,H,N,d] of the Hk heads that the H ones shared, [B,N,Hk,d]."""
    B, H, N, d = x.shape
    return x.reshape(B, Hk, H // Hk, N, d).sum(dim=2).permute(0, 2, 1, 3).contiguous().to(t)


def _run_plain(s):
    if s["op"].startswith("rotary"):
        return _run_plain_rotary(s)
    t, H, Hk, cap = TYPES[s["dtype"]], s["H"], s["Hk"], s["cap"]
    q, k, v = _heads_first(s["q"], H), _heads_first(s["k"], H), _heads_first(s["v"], H)
    z = torch.matmul(q, k.transpose(2, 3).contiguous()) * s["scale"]
    if cap:
        bent = torch.tanh(z / cap)
        z = cap * bent
    if s["slope"] is not None:
        away = s["q_xy"][:, :, None, :] - s["k_xy"][:, None, :, :]
        distance = torch.sqrt(away[..., 0] ** 2 + away[..., 1] ** 2)[:, None]
        z = z - s["slope"][:, None, None] * distance
    if s["q_doc"] is not None:
        seen = ((s["q_doc"][:, :, None] == s["k_doc"][:, None, :]) & (s["q_doc"][:, :, None] >= 0))[:, None]
        z = torch.where(seen, z, -math.inf)
    top = z.amax(dim=3, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)  # a token that sees none
    e = torch.exp(z - top)
    total = e.sum(dim=3, keepdim=True)
    p = torch.where(total > 0, e / total, 0.0)
    o = torch.matmul(p, v)
    r = {"out": o.permute(0, 2, 1, 3).contiguous().to(t), "lse": (top + torch.log(total))[..., 0].permute(0, 2, 1).contiguous()}
    if s["op"] == "attn_fwd":
        return r
    g = _heads_first(s["dout"], H)
    ds = p * (torch.matmul(g, v.transpose(2, 3).contiguous()) - (g * o).sum(dim=3, keepdim=True))
    if s["slope"] is not None:
        r["dslope"] = -(ds * distance).double().sum(dim=(0, 2, 3)).float()
    if cap:
        ds = ds * (1.0 - bent * bent)
    ds = ds * s["scale"]
    r["dq"] = torch.matmul(ds, k).permute(0, 2, 1, 3).contiguous().to(t)
    r["dk"] = _shared(torch.matmul(ds.transpose(2, 3).contiguous(), q), Hk, t)
    r["dv"] = _shared(torch.matmul(p.transpose(2, 3).contiguous(), g), Hk, t)
    return r


# ---------------------------------------------------------------------------------------------------- floors and values

def work(case):
    el = 4 if case["dtype"] == "f32" else 2
    B, H, Hk, d = (case[n] for n in ("B", "H", "Hk", "d"))
    if case["op"].startswith("rotary"):
        N, axes = case["N"], case["axes"]
        n = B * N * (H + Hk) * d
        some = 4 * (B * N * axes + d // 2 * axes)
        if case["op"] == "rotary_fwd":
            return {"bytes": 2 * n * el + some, "flops": 3 * n}
        return {"bytes": (3 if case["dcoords"] else 2) * n * el + some + (4 * B * N * axes if case["dcoords"] else 0),
                "flops": (5 if case["dcoords"] else 3) * n}
    Nq, Nk, docs = case["Nq"], case["Nk"], case["docs"]
    train, self_ = case["op"] == "attn_train", Nq == Nk
    pairs = B * Nq * Nk
    if docs:  # lengths (i + 1 + u) L - (i + v) L of a mean L, u and v uniform: their squares L^2 (1 + 1/6)
        pairs = int(pairs / docs * (63 / 64) ** 2 * (7 / 6 if docs > 1 else 1))
    n = B * d * (Nq * H * (4 if train else 2) + Nk * Hk * (4 if train else 2)) * el + 4 * B * Nq * H
    if case["distance"]:
        n += 8 * B * (Nk if self_ else Nq + Nk)
    if docs:
        n += 4 * B * (Nk if self_ else Nq + Nk)
    return {"bytes": n, "flops": (14 if train else 4) * pairs * H * d}


def _exact_rotary(case, f):
    layout, d = case["layout"], case["d"]
    c = torch.arange(d // 2, device=DEV)
    first, second = (2 * c, 2 * c + 1) if layout == "pairs" else (c, c + d // 2)
    angle = torch.einsum("bna,ca->bnc", f["coords"], f["freq"])[:, :, None]
    turn = torch.polar(torch.ones_like(angle), angle)  # pairs as complex numbers

    def pairs(x):
        return torch.complex(x[..., first], x[..., second])

    def channels(z):
        x = torch.empty(*z.shape[:-1], d, dtype=torch.float64, device=DEV)
        x[..., first], x[..., second] = z.real, z.imag
        return x

    if case["op"] == "rotary_fwd":
        return {n: channels(pairs(f[n]) * turn) for n in ("q", "k") if f[n] is not None}
    names = [n for n in ("q", "k") if f["d%s_out" % n] is not None]
    r = {"d" + n: channels(pairs(f["d%s_out" % n]) * turn.conj()) for n in names}
    if case["dcoords"]:
        spin = sum((pairs(f[n + "_out"]).conj() * pairs(f["d%s_out" % n])).imag.sum(2) for n in names)
        r["dcoords"] = torch.einsum("bnc,ca->bna", spin, f["freq"])
    return r


def exact(case, seed):
    """The same outputs from the definitions, in 64 bits: an image and a head at a time."""
    s = _inputs(case, seed)
    f = {n: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for n, v in s.items()}
    if case["op"].startswith("rotary"):
        return _exact_rotary(case, f)
    H, Hk, cap = case["H"], case["Hk"], case["cap"]
    r = {"out": torch.zeros_like(f["q"]), "lse": torch.zeros(f["q"].shape[:3], dtype=torch.float64, device=DEV)}
    if case["op"] == "attn_train":
        r.update({"d" + n: torch.zeros_like(f[n]) for n in ("q", "k", "v")})
        if case["distance"]:
            r["dslope"] = torch.zeros_like(f["slope"])
    for b in range(case["B"]):
        away = torch.cdist(f["q_xy"][b], f["k_xy"][b], compute_mode="donot_use_mm_for_euclid_dist") if case["distance"] else None
        hidden = (s["q_doc"][b][:, None] != s["k_doc"][b]) | (s["q_doc"][b][:, None] < 0) if case["docs"] else None
        for h in range(H):
            q, k, v = f["q"][b, :, h], f["k"][b, :, h * Hk // H], f["v"][b, :, h * Hk // H]
            z = f["scale"] * (q @ k.t())
            slope = None
            if cap:
                z = (z / cap).tanh()
                slope = 1 - z ** 2
                z = z * cap
            if case["distance"]:
                z = z - f["slope"][h] * away
            if case["docs"]:
                z = z.masked_fill(hidden, -math.inf)
            lse = z.logsumexp(1)
            p = (z - torch.where(lse.isinf(), 0.0, lse)[:, None]).exp()
            r["out"][b, :, h], r["lse"][b, :, h] = p @ v, lse
            if case["op"] == "attn_train":
                g = f["dout"][b, :, h]
                dp = g @ v.t()
                ds = p * (dp - (p * dp).sum(1, keepdim=True))
                if case["distance"]:
                    r["dslope"][h] -= (ds * away).sum()
                if slope is not None:
                    ds = ds * slope
                r["dq"][b, :, h] = f["scale"] * (ds @ k)
                r["dk"][b, :, h * Hk // H] += f["scale"] * (ds.t() @ q)
                r["dv"][b, :, h * Hk // H] += p.t() @ g
    return r
