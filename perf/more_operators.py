"""What the feed-forward block and dropout are timed on: the block's forward pass and gradients, dropout as a call of its own, and the
token lookup and its gradient with dropout.

`run` computes a pass in elementary torch operations, or, where `own` is set, through the package's entry points.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
K, S = 4, 5                 # data entries per parity, servers: the package's defaults
PAD = -100                  # the padding token: no row of any table
OFFSET = 3                  # the call's number among those of a step that draw masks


def listed():
    return [
        # ---- the block, forward.  A decoding step of a few sequences: the weights are what is read.
        {"name": "ffn_decode", "do": "ffn", "n": 5, "dim": 1024, "hidden": 4096, "type": "bf16", "act": "silu", "p": 0.0,
         "residual": True, "saved": False, "extra": 0},
        # a prompt in 32 bits, sizes that fit no tile, rows inside wider ones
        {"name": "ffn_odd", "do": "ffn", "n": 777, "dim": 260, "hidden": 684, "type": "f32", "act": "gelu", "p": 0.0,
         "residual": False, "saved": False, "extra": 4},
        # a training step on 64 sequences of 128 tokens of the default width
        {"name": "ffn_train", "do": "ffn", "n": 8192, "dim": 128, "hidden": 512, "type": "bf16", "act": "silu", "p": 0.1,
         "residual": True, "saved": True, "extra": 0},
        # a large training batch at the largest width of a table
        {"name": "ffn_large", "do": "ffn", "n": 16411, "dim": 1024, "hidden": 4096, "type": "bf16", "act": "silu", "p": 0.1,
         "residual": True, "saved": True, "extra": 0},
        # ---- the block, gradients of its input and weights.  Of a training step at the default width
        {"name": "ffn_grad_train", "do": "ffn_grad", "n": 8191, "dim": 128, "hidden": 512, "type": "f16", "act": "gelu", "p": 0.1,
         "residual": True, "extra": 0},
        # of a large batch
        {"name": "ffn_grad_large", "do": "ffn_grad", "n": 16411, "dim": 1024, "hidden": 4096, "type": "bf16", "act": "silu",
         "p": 0.1, "residual": True, "extra": 0},
        # ---- dropout by itself.  Of a small batch's activations: the call's latency
        {"name": "dropout_small", "do": "dropout", "n": 600, "dim": 128, "type": "bf16", "p": 0.1, "residual": False, "extra": 0},
        # of a large batch's, added to the residual stream
        {"name": "dropout_large", "do": "dropout", "n": (1 << 18) + 5, "dim": 512, "type": "bf16", "p": 0.1, "residual": True,
         "extra": 0},
        # ---- lookup with dropout.  A training step's tokens
        {"name": "embed_train", "do": "embed", "rows": 1 << 14, "dim": 128, "n": 8192, "type": "bf16", "keys": "text", "p": 0.1,
         "extra": 0},
        # a large batch of unlike tokens
        {"name": "embed_large", "do": "embed", "rows": 1 << 22, "dim": 128, "n": (1 << 20) + 77, "type": "bf16", "keys": "uniform",
         "p": 0.1, "extra": 64},
        # ---- its gradient.  A batch of text: a few tokens are most of it
        {"name": "grad_text", "do": "grad", "rows": 1 << 20, "dim": 256, "n": 1 << 16, "type": "bf16", "keys": "text", "p": 0.1,
         "extra": 0},
        # a large batch of a recommender's item ids, hardly any twice
        {"name": "grad_items", "do": "grad", "rows": 1 << 22, "dim": 128, "n": (1 << 20) + 77, "type": "f32", "keys": "uniform",
         "p": 0.2, "extra": 0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(["ffn", "ffn", "ffn_grad", "ffn_grad", "dropout", "embed", "grad"])
    kind = rng.choice(["f32", "bf16", "f16"])
    p = rng.choice([0.0, 0.1, 0.1, 0.25, 0.5])
    extra = rng.choice([0, 0, 4, 64])
    if do in ("ffn", "ffn_grad"):
        dim = 4 * _log(rng, 16, 256)
        hidden = 4 * _log(rng, max(16, dim // 8), dim)
        most = (1 << 36) if kind != "f32" else 1 << 31           # products of a projection
        n = _log(rng, 1, min(1 << 14, most // (dim * hidden)))
        case = {"do": do, "n": n, "dim": dim, "hidden": hidden, "type": kind, "act": rng.choice(["silu", "gelu", "relu"]), "p": p,
                "residual": rng.random() < 0.5, "extra": extra}
        if do == "ffn":
            case["saved"] = rng.random() < 0.5
        return case
    dim = 4 * _log(rng, 1, 256)
    n = _log(rng, 1, min(1 << 20, (1 << 27) // dim))
    if do == "dropout":
        return {"do": do, "n": n, "dim": dim, "type": kind, "p": p, "residual": rng.random() < 0.5, "extra": extra}
    rows = 4 * _log(rng, 1 << 8, min(1 << 20, (1 << 27) // dim))
    return {"do": do, "rows": rows, "dim": dim, "n": n, "type": kind, "keys": rng.choice(["text", "uniform"]),
            "p": max(p, 0.1), "extra": extra}


def _wide(case, rows, cols, dtype):
    """Room for a tensor inside wider rows."""
    return torch.zeros(rows, cols + case["extra"], dtype=dtype, device="cuda")[:, :cols]


def _random(case, rows, cols, gen, scale):
    x = _wide(case, rows, cols, TYPES[case["type"]])
    return x.copy_(torch.randn(rows, cols, generator=gen, device="cuda") * scale)


def _scale(case):
    return math.sqrt(case["dim"])


def _tokens(case, gen):
    n, rows = case["n"], case["rows"]
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    if case["keys"] == "text":          # the j-th token about 1 / j as often as the first
        keys = (torch.pow(float(rows + 1), u) - 1.0).long()
    else:
        keys = (u * rows).long()
    keys = keys.clamp_(0, rows - 1)
    return torch.where(torch.rand(n, generator=gen, device="cuda") < 0.05, torch.full_like(keys, PAD), keys)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t, n, dim, do = TYPES[case["type"]], case["n"], case["dim"], case["do"]
    # the generator's seed and the number of masks drawn before, which a program keeps on the device
    s = {"state": torch.randint(0, 1 << 62, (2,), generator=gen, device="cuda")}
    if do in ("ffn", "ffn_grad"):
        F = case["hidden"]
        s["x"] = _random(case, n, dim, gen, 1.0)
        s["gate"] = (torch.randn(F, dim, generator=gen, device="cuda") * dim ** -0.5).to(t)
        s["up"] = (torch.randn(F, dim, generator=gen, device="cuda") * dim ** -0.5).to(t)
        s["down"] = (torch.randn(dim, F, generator=gen, device="cuda") * F ** -0.5).to(t)
        if do == "ffn_grad":            # what the forward pass left, and the gradient of its output
            xs = s["x"].float()
            s["saved"] = torch.cat([xs @ s["gate"].float().t(), xs @ s["up"].float().t()], 1).to(t)
            s["d"] = _random(case, n, dim, gen, 0.1)
        elif case["residual"]:
            s["residual"] = _random(case, n, dim, gen, 1.0)
    elif do == "dropout":
        s["x"] = _random(case, n, dim, gen, 1.0)
        if case["residual"]:
            s["residual"] = _random(case, n, dim, gen, 1.0)
    else:
        s["keys"] = _tokens(case, gen)
        if do == "embed":
            s["table"] = torch.randn(case["rows"], dim, generator=gen, device="cuda") * 0.02
        else:
            s["d"] = _random(case, n, dim, gen, 0.01)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    t, n, dim, do = TYPES[case["type"]], case["n"], case["dim"], case["do"]
    if do == "grad":                    # rows behind the last distinct token are not written
        s["keys_out"] = torch.zeros(n, dtype=torch.int64, device="cuda")
        s["grads_out"] = torch.zeros(n, dim, device="cuda")
        s["count"] = torch.zeros(1, dtype=torch.int64, device="cuda")
    else:
        s["out"] = _wide(case, n, dim, t)
    if do == "ffn" and case["saved"]:
        s["saved"] = torch.zeros(n, 2 * case["hidden"], dtype=t, device="cuda")
    if do == "ffn_grad":
        s["grads"] = [torch.zeros_like(s[w]) for w in ("gate", "up", "down")]
    if not own:
        return s
    from paper_2104_01981_amd import Dropout, Ecrm, FeedForward
    s["dropout"] = Dropout(case["p"], s["state"], OFFSET) if case["p"] > 0 or do == "dropout" else None
    if do in ("ffn", "ffn_grad"):       # the block, which the program has for all its steps
        s["block"] = FeedForward(s["gate"], s["up"], s["down"], max_rows=n, activation=case["act"], training=do == "ffn_grad")
    if do in ("embed", "grad"):         # the table's context, which the program has for its updates anyway
        rows = case["rows"]
        ctx = Ecrm(rows, dim, K, S, max_batch=n)
        E = s["table"] if do == "embed" else torch.zeros(rows, dim, device="cuda")
        load = torch.zeros(2, S, dtype=torch.int64, device="cuda")
        scratch = torch.empty(ctx.scratch_bytes(), dtype=torch.uint8, device="cuda")
        ctx.bind(E, torch.zeros(rows, dim, device="cuda"), torch.zeros(rows // K, dim, device="cuda"),
                 torch.zeros(rows // K, dim, device="cuda"), load[0], load[1], scratch)
        s["ctx"] = ctx
    return s


# ---- plain form --------------------------------------------------------------------------------------------------------------
LOW = 0xFFFFFFFF


def _kept(s, rows, cols):
    """Which elements of a tensor are kept, from the seed, the mask's number, the row and eight columns at a time: Philox 4x32 with ten
    rounds (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", SC 2011), 16 bits an element; and the factor of those."""
    border = round(s["case"]["p"] * 65536)
    blocks = (cols + 7) // 8
    place = s["state"][1] + OFFSET
    i = torch.arange(rows, device="cuda")[:, None].expand(rows, blocks)
    w = [torch.arange(blocks, device="cuda")[None].expand(rows, blocks), i, (place & LOW).expand(rows, blocks),
         ((place >> 32) & LOW).expand(rows, blocks)]
    k0, k1 = s["state"][0] & LOW, (s["state"][0] >> 32) & LOW
    for _ in range(10):
        a, b = w[0] * 0xD2511F53, w[2] * 0xCD9E8D57          # modulo 2^64
        w = [((b >> 32) & LOW) ^ w[1] ^ k0, b & LOW, ((a >> 32) & LOW) ^ w[3] ^ k1, a & LOW]
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    bits = torch.stack([half for x in w for half in (x & 0xFFFF, x >> 16)], 2).view(rows, blocks * 8)[:, :cols]
    return bits >= border, 65536.0 / (65536 - border)


def _drop(s, x):
    if s["case"]["p"] == 0.0:
        return x
    kept, factor = _kept(s, x.shape[0], x.shape[1])
    return torch.where(kept, x * factor, torch.zeros((), device="cuda"))


def _activation(name, g):
    """The activation and its derivative."""
    if name == "silu":
        q = 1.0 / (1.0 + torch.exp(-g))
        return g * q, q * (1.0 + g * (1.0 - q))
    if name == "gelu":
        q = 0.5 * (1.0 + torch.erf(g * 0.5 ** 0.5))
        return g * q, q + g * torch.exp(-0.5 * g * g) * (2.0 * math.pi) ** -0.5
    positive = (g > 0).float()
    return g * positive, positive


def _plain_ffn(s, case, t):
    x = s["x"].float()
    g, u = x @ s["gate"].float().t(), x @ s["up"].float().t()
    y = _drop(s, (_activation(case["act"], g)[0] * u) @ s["down"].float().t())
    if case["residual"]:
        y = y + s["residual"].float()
    out = {"out": y.to(t)}
    if case["saved"]:
        out["saved"] = torch.cat([g, u], 1).to(t)
    return out


def _plain_ffn_grad(s, case, t):
    F, x = case["hidden"], s["x"].float()
    g, u, dy = s["saved"][:, :F].float(), s["saved"][:, F:].float(), _drop(s, s["d"].float())
    a, slope = _activation(case["act"], g)
    dh = dy @ s["down"].float()
    dg, du = dh * u * slope, dh * a
    dx = dg @ s["gate"].float() + du @ s["up"].float()
    if case["residual"]:                 # the block's input went to its output, too
        dx = dx + s["d"].float()
    return {"x": dx.to(t), "gate": (dg.t() @ x).to(t), "up": (du.t() @ x).to(t), "down": (dy.t() @ (a * u)).to(t)}


def _plain_dropout(s, case, t):
    y = _drop(s, s["x"].float())
    return (y + s["residual"].float() if case["residual"] else y).to(t)


def _plain_embed(s, case, t):
    keys = s["keys"]
    found = keys != PAD
    e = s["table"][torch.where(found, keys, torch.zeros_like(keys))] * _scale(case)
    return _drop(s, torch.where(found[:, None], e, torch.zeros((), device="cuda"))).to(t)


def _plain_grad(s, case, t):
    keys, rows, n = s["keys"], case["rows"], case["n"]
    sorted_keys, order = torch.sort(torch.where(keys == PAD, torch.full_like(keys, rows), keys), stable=True)
    real = sorted_keys < rows
    head = real.clone()
    head[1:] &= sorted_keys[1:] != sorted_keys[:-1]
    place = torch.cumsum(head, 0) - 1
    g = torch.where(real[:, None], _drop(s, s["d"].float())[order], torch.zeros((), device="cuda"))
    place = place.clamp(min=0)
    sums = torch.zeros(n, case["dim"], device="cuda").index_add_(0, place, g) * _scale(case)
    keys_out = torch.full((n + 1,), -1, dtype=torch.int64, device="cuda")
    keys_out.scatter_(0, torch.where(head, place, torch.full_like(place, n)), torch.where(head, sorted_keys, torch.full_like(keys, -1)))
    return {"keys": keys_out[:n], "grads": sums, "count": head.sum().reshape(1)}


def run(s):
    case = s["case"]
    do, drop = case["do"], s.get("dropout")
    if not own:
        return {"ffn": _plain_ffn, "ffn_grad": _plain_ffn_grad, "dropout": _plain_dropout, "embed": _plain_embed,
                "grad": _plain_grad}[do](s, case, TYPES[case["type"]])
    if do == "ffn":
        s["block"].forward(s["x"], s["out"], residual=s.get("residual"), dropout=drop, saved=s.get("saved"))
        return {"out": s["out"], "saved": s["saved"]} if case["saved"] else {"out": s["out"]}
    if do == "ffn_grad":
        gate, up, down = s["grads"]
        s["block"].backward(s["x"], s["saved"], s["d"], s["out"], gate, up, down, add=s["d"] if case["residual"] else None,
                            dropout=drop)
        return {"x": s["out"], "gate": gate, "up": up, "down": down}
    if do == "dropout":
        drop.apply(s["x"], s["out"], residual=s.get("residual"))
        return s["out"]
    if do == "embed":
        s["ctx"].embed(s["keys"], s["out"], scale=_scale(case), padding=PAD, dropout=drop)
        return s["out"]
    s["ctx"].embed_grad(s["keys"], s["d"], s["keys_out"], s["grads_out"], s["count"], scale=_scale(case), padding=PAD, dropout=drop)
    return {"keys": s["keys_out"], "grads": s["grads_out"], "count": s["count"]}


# ---- work --------------------------------------------------------------------------------------------------------------------
def _distinct(case):
    """How many different rows the tokens name, on average."""
    rows, n = case["rows"], case["n"] * 0.95
    if case["keys"] == "uniform":
        return -rows * math.expm1(n * math.log1p(-1.0 / rows))
    j = torch.arange(rows, dtype=torch.float64)
    p = torch.log((j + 2) / (j + 1)) / math.log(rows + 1)
    return float(-torch.expm1(n * torch.log1p(-p)).sum())


def work(case):
    n, dim, size, do = case["n"], case["dim"], BYTES[case["type"]], case["do"]
    if do in ("ffn", "ffn_grad"):
        weights, act = 3 * dim * case["hidden"], n * dim
        if do == "ffn":
            moved = weights + act * (3 if case["residual"] else 2) + (2 * n * case["hidden"] if case["saved"] else 0)
            return {"bytes": moved * size, "flops": 2 * n * weights}
        return {"bytes": (2 * weights + 3 * act + 2 * n * case["hidden"]) * size, "flops": 4 * n * weights}
    if do == "dropout":
        return {"bytes": n * dim * size * (3 if case["residual"] else 2), "flops": 2 * n * dim}
    distinct = _distinct(case)
    if do == "embed":
        return {"bytes": 8 * n + 4 * dim * distinct + n * dim * size, "flops": 2 * n * dim}
    return {"bytes": 8 * n + 0.95 * n * dim * size + 8 * n + distinct * 4 * dim, "flops": 2 * n * dim}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------------------
def _factors(case, state, rows, cols):
    """A mask with its factor: what each element is multiplied by."""
    if case["p"] == 0.0:
        return torch.ones((), dtype=torch.float64, device="cuda")
    border = int(math.floor(case["p"] * 65536 + 0.5))
    seed, position = int(state[0]), (int(state[1]) + OFFSET) % (1 << 64)
    shift, m32 = np.uint64(32), np.uint64(0xFFFFFFFF)
    blocks = -(-cols // 8)
    out = torch.empty(rows, cols, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 21) // blocks)
    for first in range(0, rows, step):
        last = min(rows, first + step)
        shape = (last - first, blocks)
        c0 = np.broadcast_to(np.arange(blocks, dtype=np.uint64), shape)
        c1 = np.broadcast_to(np.arange(first, last, dtype=np.uint64)[:, None], shape)
        c2 = np.full(shape, position % (1 << 32), dtype=np.uint64)
        c3 = np.full(shape, position >> 32, dtype=np.uint64)
        for r in range(10):
            key0 = np.uint64((seed + r * 0x9E3779B9) % (1 << 32))
            key1 = np.uint64(((seed >> 32) + r * 0xBB67AE85) % (1 << 32))
            left, right = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
            c0, c1, c2, c3 = (right >> shift) ^ c1 ^ key0, right & m32, (left >> shift) ^ c3 ^ key1, left & m32
        words = np.stack([c0, c1, c2, c3], -1).astype("<u4")
        halves = torch.from_numpy(words.view("<u2").reshape(last - first, 8 * blocks).astype(np.int32)).to("cuda")
        out[first:last] = (halves[:, :cols] >= border).double() * (65536.0 / (65536 - border))
    return out


def _slope(name, g):
    if name == "silu":
        return torch.sigmoid(g) + g * torch.sigmoid(g) * torch.sigmoid(-g)
    if name == "gelu":
        return 0.5 * torch.special.erfc(-g / math.sqrt(2.0)) + g * torch.exp(-g * g / 2.0) / math.sqrt(2.0 * math.pi)
    return torch.heaviside(g, torch.zeros((), dtype=torch.float64, device="cuda"))


def _value(name, g):
    if name == "silu":
        return g * torch.sigmoid(g)
    if name == "gelu":
        return 0.5 * g * torch.special.erfc(-g / math.sqrt(2.0))
    return torch.clamp(g, min=0.0)


def exact(case, seed):
    s = _inputs(case, seed)
    n, dim, do = case["n"], case["dim"], case["do"]
    m = _factors(case, s["state"], n, dim)
    if do in ("ffn", "ffn_grad"):
        F = case["hidden"]
        wg, wu, wd, x = s["gate"].double(), s["up"].double(), s["down"].double(), s["x"].double()
        if do == "ffn":
            both = torch.matmul(x, torch.cat([wg, wu]).t().contiguous())
            y = torch.matmul(_value(case["act"], both[:, :F]) * both[:, F:], wd.t().contiguous()) * m
            told = {"out": y + s["residual"].double() if case["residual"] else y}
            if case["saved"]:
                told["saved"] = both
            return told
        d = s["d"].double()
        e = d * m
        gate, up = s["saved"].double().split(F, 1)
        back = torch.matmul(e, wd)
        value = _value(case["act"], gate)
        both = torch.cat([back * _slope(case["act"], gate) * up, back * value], 1)
        dx = torch.matmul(both, torch.cat([wg, wu]))
        weights = torch.matmul(both.t().contiguous(), x)
        return {"x": dx + d if case["residual"] else dx, "gate": weights[:F], "up": weights[F:],
                "down": torch.matmul(e.t().contiguous(), value * up)}
    if do == "dropout":
        y = s["x"].double() * m
        return y + s["residual"].double() if case["residual"] else y
    at = (s["keys"] >= 0).nonzero().flatten()
    names = s["keys"][at]
    if do == "embed":
        out = torch.zeros(n, dim, dtype=torch.float64, device="cuda")
        for i in range(0, len(at), 1 << 17):
            part = at[i:i + (1 << 17)]
            out[part] = s["table"][names[i:i + (1 << 17)]].double() * _scale(case) * m[part]
        return out
    distinct, where = torch.unique(names, return_inverse=True)
    grads = torch.zeros(n, dim, dtype=torch.float64, device="cuda").index_add(0, where, s["d"][at].double() * m[at])
    return {"keys": torch.cat([distinct, distinct.new_full((n - len(distinct),), -1)]), "grads": grads * _scale(case),
            "count": torch.tensor([len(distinct)])}
