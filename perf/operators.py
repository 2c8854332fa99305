"""Layer norm, dropout and the two joined on a residual path, as measurable cases: each operator forwards and backwards, on
rows (the channels of a position side by side) and on maps (planes of pixels, as the nets of this library keep them), in fp32,
bf16 and fp16, from a handful of positions to tensors that fill the memory system.

`run` with `own = False` computes an operator from elementary torch operations in fp32; with `own = True` it makes the call of
the library's binding.  Both take the tensors that `prepare` returns.

Dropout keeps element (position q, channel c) if a 16-bit number is at least t = floor(65536 p + 1/2), and multiplies what it
keeps by 65536 / (65536 - t).  The numbers come from Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as
easy as 1, 2, 3; SC 2011) with the seed as key and (q mod 2^32, c div 8 + (q div 2^32) * 2^24, offset lo, offset hi) as counter; channel c
takes half-word c mod 8 of the four words, low half first.  A position is a row, or image * plane + pixel.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
# tensors of the activations' size that a pass reads and writes
STREAMS = {"dropout": 2, "norm": 2, "norm_grad": 3, "add_norm": 4, "add_norm_grad": 4}


def _case(name, op, layout, dtype, n, c, plane=1, p=0.0, pad=0):
    return {"name": name, "op": op, "layout": layout, "type": dtype, "n": n, "c": c, "plane": plane, "p": p, "pad": pad}


def listed():
    return [
        # dropout in front of the classes of the 512 x 512 SK net: its 200 hidden maps, fp32
        _case("dropout_maps_f32_head", "dropout", "maps", "f32", 1, 200, 512 * 512, p=0.5),
        # dropout on the 1024 maps at the bottom of the 572 x 572 U-Net: 28 x 28 pixels, latency counts
        _case("dropout_maps_bf16_bottom", "dropout", "maps", "bf16", 1, 1024, 28 * 28, p=0.5),
        # norm of a few positions, the smallest call of inference
        _case("norm_rows_bf16_few", "norm", "rows", "bf16", 16, 1024),
        # norm of the first 48 maps of the SK net (odd planes of 527 x 527), fp32
        _case("norm_maps_f32_sk", "norm", "maps", "f32", 1, 48, 527 * 527),
        # norm of many wide rows
        _case("norm_rows_bf16_many", "norm", "rows", "bf16", 65536, 2048),
        # its backward pass for a few rows of a wider buffer, channels not a multiple of eight
        _case("norm_grad_rows_f32_few", "norm_grad", "rows", "f32", 37, 777, pad=23),
        # backward pass of the norm on the 64 maps in front of the U-Net's classes, 388 x 388, four images
        _case("norm_grad_maps_bf16_unet", "norm_grad", "maps", "bf16", 4, 64, 388 * 388),
        # backward pass for ordinary rows in fp16, odd width
        _case("norm_grad_rows_f16_odd", "norm_grad", "rows", "f16", 8192, 1001),
        # residual + dropout, then norm, on the 1024 maps of the paper's inner product at 128 x 128, fp32
        _case("add_norm_maps_f32_papersk", "add_norm", "maps", "f32", 1, 1024, 128 * 128, p=0.1),
        # the same on wide rows in bf16
        _case("add_norm_rows_bf16_many", "add_norm", "rows", "bf16", 16384, 4096, p=0.1),
        # and backwards: on U-Net maps in fp16, with the gradient that reaches the sum from behind it, and on the wide rows
        _case("add_norm_grad_maps_f16_unet", "add_norm_grad", "maps", "f16", 2, 512, 52 * 52, p=0.2),
        _case("add_norm_grad_rows_bf16_many", "add_norm_grad", "rows", "bf16", 16384, 4096, p=0.1),
    ]


def draw(rng):
    op = rng.choice(sorted(STREAMS))
    layout = rng.choice(("rows", "maps"))
    dtype = rng.choice(sorted(TYPES))
    c = round(math.exp(rng.uniform(0.0, math.log(8192 if layout == "rows" else 2048))))
    elements = math.exp(rng.uniform(math.log(1 << 10), math.log(1 << 24)))
    positions = max(1, round(elements / c))
    n = positions if layout == "rows" else min(positions, rng.choice((1, 1, 2, 3, 8)))
    plane = 1 if layout == "rows" else max(1, positions // n)
    p = 0.0 if op.startswith("norm") or (op != "dropout" and rng.random() < 0.25) else round(rng.uniform(0.02, 0.7), 3)
    return {"op": op, "layout": layout, "type": dtype, "n": n, "c": c, "plane": plane, "p": p, "pad": rng.choice((0, 0, 1, 8, 13))}


def _shape(case):
    return (case["n"], case["c"]) if case["layout"] == "rows" else (case["n"], case["c"], case["plane"])


def prepare(case, seed):
    shape, pad, dtype = _shape(case), case["pad"], TYPES[case["type"]]
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    c = case["c"]
    per_channel = (1, c) if case["layout"] == "rows" else (1, c, 1)

    def normal(*size):
        return torch.randn(size, generator=gen, device=dev, dtype=torch.float32)

    def tensor(values):        # what the operators read lies in a wider buffer where pad > 0
        if not pad:
            return values.to(dtype)
        wide = torch.zeros(shape[:-1] + (shape[-1] + pad,), dtype=dtype, device=dev)
        view = wide[..., :shape[-1]]
        view.copy_(values)
        return view

    # activations: channels of unlike means and scales; those in front of dropout come out of a ReLU
    scale, shift = torch.exp(0.5 * normal(*per_channel)), normal(*per_channel)
    x = normal(*shape).mul_(scale).add_(shift)
    st = {"case": case, "seed": int(torch.randint(1 << 62, (1,), generator=gen, device=dev)), "offset": 1 + seed % 1000}
    op = case["op"]
    st["x"] = tensor(x.relu_() if op == "dropout" else x)
    del x
    st["gamma"] = 1.0 + 0.2 * normal(c)
    st["beta"] = 0.2 * normal(c)
    if op == "add_norm":
        st["residual"] = tensor(2.0 * normal(*shape))
    if op.endswith("grad"):    # x is what was normalised, with the statistics that the forward pass leaves
        wide = st["x"].double()
        mean = wide.mean(1)
        rstd = torch.rsqrt(wide.var(1, unbiased=False) + EPS)
        del wide
        st["mean"], st["rstd"] = mean.float(), rstd.float()
        st["dy"] = tensor(0.01 * normal(*shape))
        st["dgamma"], st["dbeta"] = torch.empty_like(st["gamma"]), torch.empty_like(st["beta"])
    if op == "add_norm_grad":
        st["dsum"] = tensor(0.01 * normal(*shape))

    def empty():
        return torch.empty(shape, dtype=dtype, device=dev)

    st["out"] = empty()
    if op.startswith("add_norm"):
        st["out2"] = empty()
    if op in ("norm", "add_norm"):
        st["mean"] = torch.empty((case["n"], case["plane"])[:len(shape) - 1], dtype=torch.float32, device=dev)
        st["rstd"] = torch.empty_like(st["mean"])
    return st


# ---- the plain form -----------------------------------------------------------------------------------------------

def _keep_scale(case, seed, offset, device):
    """[n, c(, plane)] fp32: what dropout multiplies by, 0 where it drops (bits in int64, 32 at a time)."""
    c, positions = case["c"], case["n"] * case["plane"]
    t = int(case["p"] * 65536.0 + 0.5)
    if t >= 65536:
        return torch.zeros(_shape(case), device=device)
    groups = (c + 7) // 8
    low = 0xFFFFFFFF
    q = torch.arange(positions, dtype=torch.int64, device=device)[:, None]
    g = torch.arange(groups, dtype=torch.int64, device=device)[None, :]
    w0 = (q & low).expand(positions, groups)
    w1 = g | ((q >> 32) << 24)
    w2 = torch.full_like(w1, offset & low)
    w3 = torch.full_like(w1, offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = w0 * 0xD2511F53, w2 * 0xCD9E8D57          # modulo 2^64; the shifts' copies of the sign are masked away
        w0, w1, w2, w3 = ((b >> 32) & low) ^ w1 ^ k0, b & low, ((a >> 32) & low) ^ w3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    fields = torch.stack([half for w in (w0, w1, w2, w3) for half in (w & 0xFFFF, w >> 16)], dim=2).reshape(positions, groups * 8)[:, :c]
    keep = (fields >= t).to(torch.float32) * (65536.0 / (65536 - t))
    if case["layout"] == "rows":
        return keep
    return keep.reshape(case["n"], case["plane"], c).transpose(1, 2)


def _dropped(case, st, values):
    if case["p"] == 0.0:
        return values
    keep = _keep_scale(case, st["seed"], st["offset"], values.device)
    return torch.where(keep > 0, values * keep, torch.zeros_like(values))


def _plain(st):
    case = st["case"]
    op, dtype = case["op"], TYPES[case["type"]]
    x = st["x"].float()
    if op == "dropout":
        return _dropped(case, st, x).to(dtype)
    along = [1, -1] + [1] * (x.dim() - 2)                # gamma and beta on the axis of the channels
    gamma = st["gamma"].reshape(along)
    if op in ("norm", "add_norm"):
        s = x if op == "norm" else st["residual"].float() + _dropped(case, st, x)
        mean = s.mean(1, keepdim=True)
        d = s - mean
        rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
        y = (d * rstd * gamma + st["beta"].reshape(along)).to(dtype)
        out = [y, mean.squeeze(1), rstd.squeeze(1)]
        return out if op == "norm" else out + [s.to(dtype)]
    dy = st["dy"].float()
    rstd = st["rstd"].unsqueeze(1)
    h = (x - st["mean"].unsqueeze(1)) * rstd
    g = dy * gamma
    ds = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    others = [0] + list(range(2, x.dim()))
    sums = [(dy * h).sum(others), dy.sum(others)]
    if op == "norm_grad":
        return [ds.to(dtype)] + sums
    ds = ds + st["dsum"].float()
    return [_dropped(case, st, ds).to(dtype), ds.to(dtype)] + sums


# ---- the library's calls ------------------------------------------------------------------------------------------

def _own(st):
    from paper_1509_03371_amd import binding as B
    case = st["case"]
    op, p, seed, offset = case["op"], case["p"], st["seed"], st["offset"]
    if op == "dropout":
        return B.dropout(st["x"], p, seed, offset, axis=1, out=st["out"])
    if op == "norm":
        y, _, mean, rstd = B.layer_norm(st["x"], st["gamma"], st["beta"], EPS, axis=1, out=st["out"], mean=st["mean"], rstd=st["rstd"])
        return [y, mean, rstd]
    if op == "add_norm":
        y, s, mean, rstd = B.layer_norm(st["x"], st["gamma"], st["beta"], EPS, axis=1, residual=st["residual"], p=p, seed=seed, offset=offset,
                                        out=st["out"], sum_out=st["out2"], mean=st["mean"], rstd=st["rstd"])
        return [y, mean, rstd, s]
    if op == "norm_grad":
        dx, _, dgamma, dbeta = B.layer_norm_backward(st["dy"], st["x"], st["mean"], st["rstd"], st["gamma"], axis=1, dx=st["out"],
                                                     dgamma=st["dgamma"], dbeta=st["dbeta"])
        return [dx, dgamma, dbeta]
    dx, dres, dgamma, dbeta = B.layer_norm_backward(st["dy"], st["x"], st["mean"], st["rstd"], st["gamma"], axis=1, dsum=st["dsum"], p=p, seed=seed,
                                                    offset=offset, dx=st["out"], dresidual=st["out2"] if p > 0.0 else None,
                                                    dgamma=st["dgamma"], dbeta=st["dbeta"])
    return [dx, dres, dgamma, dbeta]


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    op = case["op"]
    elements, positions = case["n"] * case["c"] * case["plane"], case["n"] * case["plane"]
    streams = STREAMS[op] + (1 if op == "add_norm_grad" and case["p"] > 0.0 else 0)
    channels = {"dropout": 0, "norm": 2, "add_norm": 2}.get(op, 3)       # gamma, beta; gamma, dgamma, dbeta
    nbytes = streams * elements * SIZE[case["type"]] + (0 if op == "dropout" else 8 * positions) + 4 * channels * case["c"]
    flops = {"dropout": 1, "norm": 8, "add_norm": 10, "norm_grad": 14, "add_norm_grad": 16}[op] * elements
    return {"bytes": nbytes, "flops": flops}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------

def _mask64(case, seed, offset):
    """Which elements dropout keeps, positions x channels, by numpy's unsigned 64-bit products."""
    positions, c = case["n"] * case["plane"], case["c"]
    groups = -(-c // 8)
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    ctr = np.empty((4, positions, groups), np.uint64)
    q = np.arange(positions, dtype=np.uint64)[:, None]
    ctr[0] = q & low
    ctr[1] = np.arange(groups, dtype=np.uint64)[None, :] + (q >> half) * np.uint64(1 << 24)
    ctr[2] = offset % (1 << 32)
    ctr[3] = offset // (1 << 32)
    key = [seed % (1 << 32), seed // (1 << 32)]
    for _ in range(10):
        left, right = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
        ctr[0] = (right >> half) ^ ctr[1] ^ np.uint64(key[0])
        ctr[1] = right & low
        ctr[2] = (left >> half) ^ ctr[3] ^ np.uint64(key[1])
        ctr[3] = left & low
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    numbers = np.ascontiguousarray(ctr.transpose(1, 2, 0).astype("<u4")).view("<u2").reshape(positions, groups * 8)[:, :c]
    return numbers >= math.floor(65536 * case["p"] + 0.5)


def exact(case, seed):
    st = prepare(case, seed)
    op, c = case["op"], case["c"]
    maps = case["layout"] == "maps"

    def by_position(t):        # positions x channels, in 64 bits
        t = t.to(torch.float64)
        return t.permute(0, 2, 1).reshape(-1, c) if maps else t

    def as_given(t):
        return t.reshape(case["n"], case["plane"], c).permute(0, 2, 1).contiguous() if maps else t

    def per_position(t):
        return t.reshape(case["n"], case["plane"]) if maps else t.reshape(-1)

    def drop(t):
        if case["p"] == 0.0:
            return t
        kept = torch.from_numpy(_mask64(case, st["seed"], st["offset"])).to(t.device)
        t = t * (65536.0 / (65536 - math.floor(65536 * case["p"] + 0.5)))
        return t.masked_fill_(~kept, 0.0)

    x = by_position(st["x"])
    if op == "dropout":
        return as_given(drop(x))
    gamma, beta = st["gamma"].double(), st["beta"].double()
    if not op.endswith("grad"):
        if op == "add_norm":
            x = drop(x) + by_position(st["residual"])
        mu = x.sum(1, keepdim=True) / c
        centred = x - mu
        r = 1.0 / ((centred ** 2).sum(1, keepdim=True) / c + EPS).sqrt()
        out = [as_given(centred * r * gamma + beta), per_position(mu), per_position(r)]
        return out + [as_given(x)] if op == "add_norm" else out
    dy = by_position(st["dy"])
    r = st["rstd"].double().reshape(-1, 1)
    h = (x - st["mean"].double().reshape(-1, 1)) * r
    weighted = dy * gamma
    ds = weighted - weighted.sum(1, keepdim=True) / c - h * ((weighted * h).sum(1, keepdim=True) / c)
    ds = ds * r
    sums = [(dy * h).sum(0), dy.sum(0)]
    if op == "norm_grad":
        return [as_given(ds)] + sums
    ds = ds + by_position(st["dsum"])
    res = as_given(ds)
    return [as_given(drop(ds.clone())), res] + sums
