"""The dense half of a block as a program that uses this library has it done: matrix product with its epilogue, group norm with
an activation (layer norm among it), and dropout from a counter-based generator, each forward and backward.

A case is a dict of plain values.  `op` names the call of one pass:

  linear_fwd    out = residual + dropout(act(x W^T + bias)); `pre` also returns x W^T + bias, which the backward reads
  linear_bwd    dx, dW and dbias from dout (and pre, where there is an activation)
  norm_fwd      out = act(gamma * (x - mean) * rstd + beta) over x [B,N,C], mean and rstd per image and group of channels;
                B tokens of N = 1 and one group are the layer norm of every token
  norm_bwd      dx, dgamma and dbeta
  dropout_fwd   out = residual + dropout(x)
  dropout_bwd   dx = dropout(dout)

dropout(v) of element i (in the order of memory) is 0 where the generator's word for i is below floor(p * 2^32), else v / (1 - p).
The words are those of Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011):
key = the seed, counter = (i / 4, call number), word i % 4.

Where `own` is false `run` computes the operators with elementary torch operations in 32 bits.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------------- the cases

def _linear(name, op, dtype, rows, cin, cout, act="none", p=0.0, bias=True, residual=False, pre=False):
    c = {"op": op, "dtype": dtype, "rows": rows, "cin": cin, "cout": cout, "act": act, "p": p, "bias": bias,
         "residual": residual, "pre": pre}
    if name:
        c["name"] = name
    return c


def _norm(name, op, dtype, B, N, C, groups, act="none", affine=True):
    c = {"op": op, "dtype": dtype, "B": B, "N": N, "C": C, "groups": groups, "act": act, "affine": affine}
    if name:
        c["name"] = name
    return c


def _dropout(name, op, dtype, rows, C, p, residual=False):
    c = {"op": op, "dtype": dtype, "rows": rows, "C": C, "p": p, "residual": residual}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one image of 256 tokens in fp32, first product of the block's MLP: latency counts
        _linear("linear_tiny", "linear_fwd", "f32", 256, 64, 192, act="gelu", pre=True),
        # fine-tuning on 1024-px images, first stage, 8 images of 16384 tokens: first product of the MLP (ratio 3), in training
        _linear("linear_up_finetune", "linear_fwd", "bf16", 131072, 64, 192, act="gelu", pre=True),
        # a merged stage, 64 images of 1024 tokens: the product behind the attention, with dropout, onto the residual stream
        _linear("linear_out_merged", "linear_fwd", "bf16", 65536, 256, 256, p=0.1, residual=True),
        # inference on a single small image in the last stage: 64 tokens, the MLP's second product onto the residual stream
        _linear("linear_few_rows", "linear_fwd", "bf16", 64, 2304, 768, residual=True),
        # the largest: training of a wide stage, gradients of the MLP's first product
        _linear("linear_bwd_wide", "linear_bwd", "bf16", 16384, 768, 2304, act="gelu"),
        # whatever sizes a head has, in full precision: rows of no whole 16 bytes, with dropout behind the activation
        _linear("linear_bwd_ragged", "linear_bwd", "f32", 12003, 100, 301, act="silu", p=0.2),
        # layer norm in front of the attention, first stage of fine-tuning
        _norm("layer_norm_finetune", "norm_fwd", "bf16", 131072, 1, 64, 1),
        # its gradients in a merged stage
        _norm("layer_norm_bwd_merged", "norm_bwd", "bf16", 65536, 1, 256, 1),
        # group norm and activation between the layers of a head on full-resolution token maps, full precision
        _norm("group_norm_head", "norm_fwd", "f32", 8, 16384, 64, 8, act="silu"),
        # its gradients on what a mask leaves: a small batch, token counts that nothing divides
        _norm("group_norm_bwd_ragged", "norm_bwd", "bf16", 3, 4001, 96, 12, act="relu"),
        # dropout of a branch onto the residual stream, 16 images of 16384 tokens
        _dropout("dropout_residual", "dropout_fwd", "bf16", 262144, 128, 0.1, residual=True),
        # backward of a small one, of no whole 16 bytes
        _dropout("dropout_bwd_small", "dropout_bwd", "f32", 257, 63, 0.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear_fwd", "linear_fwd", "linear_bwd", "linear_bwd", "norm_fwd", "norm_bwd", "dropout_fwd", "dropout_bwd"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    act = rng.choice(["none", "relu", "gelu", "silu"])
    p = rng.choice([0.0, 0.0, 0.1, rng.uniform(0.01, 0.9)])
    if op.startswith("linear"):
        cin, cout = (rng.choice([c, c // 8 * 8 or c, c // 64 * 64 or c]) for c in (_log(rng, 3, 2304), _log(rng, 1, 2304)))
        most = 2.5e10 if dtype == "bf16" else 2.5e9  # a fraction of the largest listed case's products
        rows = max(1, min(_log(rng, 1, 131072), int(most / (cin * cout)), int(3e7 / max(cin, cout))))
        return _linear(None, op, dtype, rows, cin, cout, act, p, bias=rng.random() < 0.8,
                       residual=op == "linear_fwd" and rng.random() < 0.5, pre=op == "linear_fwd" and rng.random() < 0.5)
    if op.startswith("norm"):
        if rng.random() < 0.5:  # of every token
            C = _log(rng, 16, 2304)
            C = rng.choice([C, C // 8 * 8])
            return _norm(None, op, dtype, min(_log(rng, 1, 131072), int(3e7 / C)), 1, C, 1, act, rng.random() < 0.9)
        groups = rng.choice([1, 2, 4, 8, 16, 32, rng.randint(1, 24)])
        C = groups * rng.choice([1, 2, 4, 8, 8, 16, rng.randint(1, 40)])
        N = _log(rng, 2, 16384)
        B = max(1, min(_log(rng, 1, 64), int(3e7 / (C * N))))
        return _norm(None, op, dtype, B, N, C, groups, act, rng.random() < 0.9)
    C = _log(rng, 1, 2304)
    C = rng.choice([C, C // 8 * 8 or C])
    return _dropout(None, op, dtype, min(_log(rng, 1, 262144), int(3e7 / C)), C, p or 0.25, op == "dropout_fwd" and rng.random() < 0.5)


# --------------------------------------------------------------------------------------------------------- their inputs

def _inputs(case, seed):
    """The tensors that the call reads, from the seed alone."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t = TYPES[case["dtype"]]

    def normal(*shape, std=1.0, mean=0.0):
        return (torch.randn(shape, generator=g, device=DEV) * std + mean).to(t)

    d = {}
    if case["op"].startswith("linear"):
        rows, cin, cout = case["rows"], case["cin"], case["cout"]
        d["x"] = normal(rows, cin)                              # normalised tokens
        d["weight"] = normal(cout, cin, std=cin ** -0.5)        # as initialised: outputs of unit variance
        if case["op"] == "linear_fwd":
            d["bias"] = normal(cout, std=0.2) if case["bias"] else None
            d["residual"] = normal(rows, cout, std=2.0) if case["residual"] else None
        else:
            d["dout"] = normal(rows, cout)
            d["pre"] = normal(rows, cout, std=1.1) if case["act"] != "none" else None
    elif case["op"].startswith("norm"):
        B, N, C, G = case["B"], case["N"], case["C"], case["groups"]
        # a residual stream: channels with offsets and scales of their own
        spread = torch.rand(C, generator=g, device=DEV) * 1.5 + 0.5
        shift = torch.randn(C, generator=g, device=DEV) * 0.7
        d["x"] = (torch.randn(B, N, C, generator=g, device=DEV) * spread + shift).to(t)
        d["gamma"] = normal(C, std=0.2, mean=1.0) if case["affine"] else None
        d["beta"] = normal(C, std=0.2) if case["affine"] else None
        if case["op"] == "norm_bwd":
            d["dout"] = normal(B, N, C)
            v = d["x"].double().reshape(B, N, G, C // G)
            mean = v.mean(dim=(1, 3))
            var = ((v - mean[:, None, :, None]) ** 2).mean(dim=(1, 3))
            d["mean"] = mean.float()
            d["rstd"] = (1.0 / (var + EPS).sqrt()).float()
    else:
        name = "x" if case["op"] == "dropout_fwd" else "dout"
        d[name] = normal(case["rows"], case["C"])
        if case["op"] == "dropout_fwd":
            d["residual"] = normal(case["rows"], case["C"], std=2.0) if case["residual"] else None
    # (seed, call number) of the generator, in device memory, as a program keeps them from step to step
    d["rng"] = torch.tensor([seed * 7919 + 12345, 3 + seed % 1000], dtype=torch.int64, device=DEV)
    return d


EPS = 1e-5


def prepare(case, seed):
    s = dict(case)
    s.update(_inputs(case, seed))
    return s


# -------------------------------------------------------------------------------------------------- one pass, both ways

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2602_16249_amd as aff
    op = s["op"]
    rng = s["rng"] if s.get("p") else None
    if op == "linear_fwd":
        out, pre = aff.affmae_linear_fwd(s["x"], s["weight"], s["bias"], s["residual"], act=s["act"], p=s["p"], rng=rng,
                                         want_pre=s["pre"])
        return {"out": out, "pre": pre} if s["pre"] else {"out": out}
    if op == "linear_bwd":
        return aff.affmae_linear_bwd(s["x"], s["weight"], s["dout"], s["pre"], act=s["act"], p=s["p"], rng=rng,
                                     want_dbias=s["bias"])
    if op == "norm_fwd":
        out, mean, rstd = aff.affmae_norm_fwd(s["x"], s["gamma"], s["beta"], s["groups"], EPS, act=s["act"])
        return {"out": out, "mean": mean, "rstd": rstd}
    if op == "norm_bwd":
        return aff.affmae_norm_bwd(s["x"], s["gamma"], s["beta"], s["mean"], s["rstd"], s["dout"], s["groups"], act=s["act"])
    if op == "dropout_fwd":
        return {"out": aff.affmae_dropout_fwd(s["x"], s["p"], rng, residual=s["residual"])}
    return {"dx": aff.affmae_dropout_bwd(s["dout"], s["p"], rng)}


LOW = 0xFFFFFFFF


def _words(count, rng):
    """The generator's words of elements 0 .. count-1, in 64-bit integers.  (A 32 x 32-bit product's high word is the wrapped
    64-bit product shifted right and masked, whatever its sign.)"""
    i = torch.arange((count + 3) // 4, device=rng.device, dtype=torch.int64)
    k0, k1 = rng[0] & LOW, (rng[0] >> 32) & LOW
    c0, c1 = i & LOW, i >> 32
    c2, c3 = (rng[1] & LOW).expand_as(i), ((rng[1] >> 32) & LOW).expand_as(i)
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & LOW) ^ c1 ^ k0, b & LOW, ((a >> 32) & LOW) ^ c3 ^ k1, a & LOW
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    return torch.stack((c0, c1, c2, c3), dim=1).reshape(-1)[:count]


def _threshold(p):
    """(words below this are dropped, factor of the others), of p as the fp32 value that the call takes"""
    p = float(torch.tensor(p, dtype=torch.float32))
    return math.floor(p * 4294967296.0), 1.0 / (1.0 - p)


def _dropped(v, p, rng):
    if not p:
        return v
    least, factor = _threshold(p)
    keep = _words(v.numel(), rng).reshape(v.shape) >= least
    return torch.where(keep, v * factor, torch.zeros_like(v))


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * 0.7071067811865476))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _dact(z, act):
    if act == "relu":
        return torch.where(z > 0, torch.ones_like(z), torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * 0.7071067811865476)) + z * torch.exp(-0.5 * z * z) * 0.3989422804014327
    if act == "silu":
        sg = 1.0 / (1.0 + torch.exp(-z))
        return sg * (1.0 + z * (1.0 - sg))
    return torch.ones_like(z)


def _run_plain(s):
    op, t = s["op"], TYPES[s["dtype"]]
    if op == "linear_fwd":
        z = s["x"].float() @ s["weight"].float().t().contiguous()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        out = _dropped(_act(z, s["act"]), s["p"], s["rng"])
        if s["residual"] is not None:
            out = s["residual"].float() + out
        return {"out": out.to(t), "pre": z.to(t)} if s["pre"] else {"out": out.to(t)}
    if op == "linear_bwd":
        dz = _dropped(s["dout"].float(), s["p"], s["rng"])
        if s["pre"] is not None:
            dz = dz * _dact(s["pre"].float(), s["act"])
        g = {"dx": (dz @ s["weight"].float()).to(t), "dweight": (dz.t().contiguous() @ s["x"].float()).to(t)}
        if s["bias"]:
            g["dbias"] = dz.sum(dim=0).to(t)
        return g
    if op == "norm_fwd":
        B, N, C = s["x"].shape
        v = s["x"].float().reshape(B, N, s["groups"], C // s["groups"])
        mean = v.mean(dim=(1, 3))
        c = v - mean[:, None, :, None]
        rstd = 1.0 / torch.sqrt((c * c).mean(dim=(1, 3)) + EPS)
        z = (c * rstd[:, None, :, None]).reshape(B, N, C)
        if s["gamma"] is not None:
            z = z * s["gamma"].float() + s["beta"].float()
        return {"out": _act(z, s["act"]).to(t), "mean": mean, "rstd": rstd}
    if op == "norm_bwd":
        B, N, C = s["x"].shape
        G = s["groups"]
        rstd = s["rstd"][:, None, :, None]
        xhat = ((s["x"].float().reshape(B, N, G, C // G) - s["mean"][:, None, :, None]) * rstd).reshape(B, N, C)
        dz = s["dout"].float()
        z = xhat if s["gamma"] is None else xhat * s["gamma"].float() + s["beta"].float()
        dz = dz * _dact(z, s["act"])
        dxhat = dz if s["gamma"] is None else dz * s["gamma"].float()
        dxhat4, xhat4 = dxhat.reshape(B, N, G, C // G), xhat.reshape(B, N, G, C // G)
        m1 = dxhat4.mean(dim=(1, 3), keepdim=True)
        m2 = (dxhat4 * xhat4).mean(dim=(1, 3), keepdim=True)
        dx = (rstd * (dxhat4 - m1 - xhat4 * m2)).reshape(B, N, C)
        if s["gamma"] is None:
            return {"dx": dx.to(t)}
        return {"dx": dx.to(t), "dgamma": (dz * xhat).sum(dim=(0, 1)), "dbeta": dz.sum(dim=(0, 1))}
    if op == "dropout_fwd":
        out = _dropped(s["x"].float(), s["p"], s["rng"])
        if s["residual"] is not None:
            out = s["residual"].float() + out
        return {"out": out.to(t)}
    return {"dx": _dropped(s["dout"].float(), s["p"], s["rng"]).to(t)}


# ---------------------------------------------------------------------------------------------------- floors and values

def work(case):
    el = 4 if case["dtype"] == "f32" else 2
    if case["op"].startswith("linear"):
        M, K, N = case["rows"], case["cin"], case["cout"]
        if case["op"] == "linear_fwd":
            n = M * K + N * K + M * N * (1 + case["residual"] + case["pre"]) + (N if case["bias"] else 0)
            return {"bytes": n * el, "flops": 2 * M * K * N}
        n = 2 * (M * K + N * K) + M * N * (2 if case["act"] != "none" else 1) + (N if case["bias"] else 0)
        return {"bytes": n * el, "flops": 4 * M * K * N}
    if case["op"].startswith("norm"):
        n, C = case["B"] * case["N"] * case["C"], case["C"] if case["affine"] else 0
        stats = case["B"] * case["groups"] * 2 * 4
        if case["op"] == "norm_fwd":
            return {"bytes": (2 * n + 2 * C) * el + stats, "flops": 8 * n}
        return {"bytes": (3 * n + 2 * C) * el + 8 * C + stats, "flops": 14 * n}
    n = case["rows"] * case["C"]
    return {"bytes": n * el * (3 if case["residual"] else 2), "flops": 2 * n}


def _exact_keep(shape, p, rng):
    """Truth of `the element stays`, by numpy's unsigned 64-bit integers on the host, a column of counters at a time."""
    import numpy as np
    seed, call = (int(v) & 0xFFFFFFFFFFFFFFFF for v in rng.tolist())
    count = math.prod(shape)
    p32 = float(np.float32(p))
    least = np.uint64(int(p32 * 2.0 ** 32))
    mask, half = np.uint64(LOW), np.uint64(32)
    keep = np.empty(((count + 3) // 4, 4), dtype=bool)
    step = 1 << 20
    for at in range(0, keep.shape[0], step):
        i = np.arange(at, min(at + step, keep.shape[0]), dtype=np.uint64)
        x = [i & mask, i >> half, np.full_like(i, call & LOW), np.full_like(i, call >> 32)]
        k0, k1 = seed & LOW, seed >> 32
        for _ in range(10):
            lo, hi = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
            x = [(hi >> half) ^ x[1] ^ np.uint64(k0), hi & mask, (lo >> half) ^ x[3] ^ np.uint64(k1), lo & mask]
            k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
        for w in range(4):
            keep[at:at + step, w] = x[w] >= least
    return torch.from_numpy(keep.reshape(-1)[:count].reshape(shape)).to(DEV), 1.0 / (1.0 - p32)


def exact(case, seed):
    """The same outputs from the definitions, in 64 bits: derivatives of the activations by their own formulas, statistics as
    sums over each group's values."""
    d = _inputs(case, seed)
    f = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in d.items()}
    keep = None
    if case.get("p"):
        shape = (case["rows"], case.get("cout", case.get("C")))
        keep, factor = _exact_keep(shape, case["p"], d["rng"])
    act = case.get("act", "none")

    def value(z):
        if act == "gelu":
            return z * 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
        return {"none": lambda v: v, "relu": lambda v: v.clamp(min=0.0), "silu": lambda v: v * torch.sigmoid(v)}[act](z)

    def slope(z):
        if act == "gelu":
            return 0.5 * torch.special.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
        if act == "silu":
            sg = torch.sigmoid(z)
            return sg + z * sg * torch.sigmoid(-z)
        return (z > 0).double() if act == "relu" else torch.ones_like(z)

    def drop(v):
        return v if keep is None else torch.where(keep, v * factor, 0.0)

    op = case["op"]
    if op == "linear_fwd":
        z = torch.mm(f["x"], f["weight"].t())
        if f["bias"] is not None:
            z += f["bias"]
        out = drop(value(z))
        out = out if f["residual"] is None else out + f["residual"]
        return {"out": out, "pre": z} if case["pre"] else {"out": out}
    if op == "linear_bwd":
        dz = drop(f["dout"])
        dz = dz if f["pre"] is None else dz * slope(f["pre"])
        g = {"dx": torch.mm(dz, f["weight"]), "dweight": torch.mm(dz.t(), f["x"])}
        if case["bias"]:
            g["dbias"] = dz.sum(0)
        return g
    if op.startswith("norm"):
        B, N, C, G = case["B"], case["N"], case["C"], case["groups"]
        x = f["x"].view(B, N, G, C // G).transpose(1, 2).reshape(B, G, -1)  # every group's values side by side
        n = x.shape[2]

        def back(v):
            return v.view(B, G, N, C // G).transpose(1, 2).reshape(B, N, C)

        if op == "norm_fwd":
            mean = x.sum(2) / n
            var = ((x - mean[..., None]) ** 2).sum(2) / n
            rstd = (var + EPS) ** -0.5
            z = back((x - mean[..., None]) * rstd[..., None])
            z = z if f["gamma"] is None else z * f["gamma"] + f["beta"]
            return {"out": value(z), "mean": mean, "rstd": rstd}
        xhat = (x - f["mean"][..., None]) * f["rstd"][..., None]
        z = back(xhat)
        dz = f["dout"] * slope(z if f["gamma"] is None else z * f["gamma"] + f["beta"])
        dh = dz if f["gamma"] is None else dz * f["gamma"]
        dh = dh.view(B, N, G, C // G).transpose(1, 2).reshape(B, G, -1)
        dx = f["rstd"][..., None] * (dh - dh.sum(2, keepdim=True) / n - xhat * (dh * xhat).sum(2, keepdim=True) / n)
        g = {"dx": back(dx)}
        if f["gamma"] is not None:
            g["dgamma"], g["dbeta"] = (dz * z).sum((0, 1)), dz.sum((0, 1))
        return g
    v = drop(f["x"] if op == "dropout_fwd" else f["dout"])
    if op == "dropout_fwd":
        return {"out": v if f["residual"] is None else v + f["residual"]}
    return {"dx": v}
