"""What stands around the block: the layers of a text encoder that turn a prompt into the tokens which cross-attention reads, and
projections in 8-bit integers, as cases that can be timed and compared.

Attention whose logits get a learned bias by the bucket of the distance between query and key (`attention`), the gated half of a
feed-forward block (`gated`), both with their gradients for adapting an encoder, and a projection whose tokens are quantised and
multiplied with weights of 8-bit integers, a scale for each token and output channel (`linear8`).

`own` false: `run` computes the operators from elementary torch operations in 32 bits; true: by the library's calls. `exact` has the
same results in 64 bits, written from the definitions.
"""
import math

import torch

own = False

DEV = "cuda"
BF = torch.bfloat16


def listed():
    return [
        # the timestep's embedding to the modulations of a block of width 5120: one token, bound by reading the weights
        _linear8("linear8_token", 1, 30720, 5120, "bf16"),
        # a prompt's 512 tokens of width 4096 to a width of 1536, as the framework projects its text
        _linear8("linear8_text", 512, 1536, 4096, "gelu"),
        # the tokens of a region step through the second half of a feed-forward block, fp32 results for the residual; ragged rows
        _linear8("linear8_region", 13103, 1536, 8960, "f32"),
        # all tokens of a 480p clip through the first half
        _linear8("linear8_clip", 32760, 8960, 1536, "gelu"),
        # one token of an encoder of width 4096: bound by reading the weights
        _gated("gated_token", 1, 10240, 4096, "gelu", False),
        # a prompt padded to 512 tokens
        _gated("gated_prompt", 512, 10240, 4096, "gelu", False),
        # 77 tokens of a small model, with the gradients: launches and latency
        _gated("gated_train_small", 77, 1024, 256, "silu", True),
        # eight prompts of 512 tokens, with the gradients
        _gated("gated_train", 4096, 10240, 4096, "gelu", True),
        # a decoder's next token over caches of different lengths: few rows, a long axis
        _attention("attn_token", 4, 64, 64, 64, 1, 4097, causal=True, ragged=True),
        # two prompts of different lengths, padded to 512 tokens, 64 heads
        _attention("attn_prompt", 2, 64, 64, 64, 512, 512, ragged=True),
        # eight such prompts, with the gradients
        _attention("attn_train", 8, 64, 64, 64, 512, 512, ragged=True, train=True),
        # one long text, wide heads that share keys, with the gradients
        _attention("attn_train_long", 1, 12, 4, 128, 8191, 8191, train=True, scale=128 ** -0.5),
    ]


def _linear8(name, M, N, K, epilogue):
    return {"name": name, "kind": "linear8", "M": M, "N": N, "K": K, "epilogue": epilogue}


def _gated(name, M, F, K, act, train):
    return {"name": name, "kind": "gated", "M": M, "F": F, "K": K, "act": act, "train": train}


def _attention(name, B, H, Hk, dh, Lq, Lk, causal=False, ragged=False, empty=False, train=False, scale=1.0, buckets=32, far=128):
    """scale: the factor of the product of query and key; buckets, far: rows of the table, distance from which on all share a bucket;
    ragged: sequences of different lengths; empty: the last one has no keys."""
    return {"name": name, "kind": "attention", "B": B, "H": H, "Hk": Hk, "dh": dh, "Lq": Lq, "Lk": Lk, "causal": causal, "ragged": ragged,
            "empty": empty, "train": train, "scale": scale, "buckets": buckets, "far": far}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear8", "gated", "attention"])
    if kind == "linear8":
        N, K = 8 * _log(rng, 1, 1920), 8 * _log(rng, 8, 1728)
        M = max(1, min(_log(rng, 1, 32760), 32760 * 8960 * 1536 // (N * K)))
        c = _linear8(None, M, N, K, rng.choice(["bf16", "gelu", "f32"]))
    elif kind == "gated":
        F, K = 64 * _log(rng, 1, 216), 64 * _log(rng, 1, 80)
        train = rng.random() < 0.5
        M = max(1, min(_log(rng, 1, 8192), 4096 * 10240 * 4096 // (F * K)))
        c = _gated(None, M, F, K, rng.choice(["gelu", "silu"]), train)
    else:
        dh = rng.choice([64, 128])
        H = rng.choice([1, 3, 4, 8, 12, 16, 32, 64])
        Hk = rng.choice([h for h in (1, 2, 4, H) if H % h == 0]) if rng.random() < 0.3 else H
        B = rng.choice([1, 1, 2, 3, 5, 8])
        train = rng.random() < 0.5
        Lk = _log(rng, 1, 8192)
        Lq = Lk if train or rng.random() < 0.5 else _log(rng, 1, 64)
        while B * H * dh * Lq * Lk > 12 * 128 * 8191 ** 2:
            Lk, Lq = -(-Lk // 2), -(-Lq // 2)
        buckets = rng.choice([8, 16, 32, 32, 64])
        c = _attention(None, B, H, Hk, dh, Lq, Lk, rng.random() < 0.4, rng.random() < 0.5, B > 1 and rng.random() < 0.2, train,
                       rng.choice([1.0, dh ** -0.5]), buckets, rng.choice([buckets, 128, rng.randint(buckets, 512)]))
    c.pop("name")
    return c


# ------------------------------------------------------------------------------------------------ inputs

class _Gen:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed))

    def normal(self, shape, std=1.0, dtype=torch.float32):
        t = torch.empty(shape, dtype=torch.float32, device=DEV)
        t.normal_(0.0, std, generator=self.g)
        return t.to(dtype)

    def uniform(self, shape):
        return torch.rand(shape, generator=self.g, device=DEV)


def _lengths(case):
    """Keys of each sequence."""
    B, Lk = case["B"], case["Lk"]
    lens = [Lk - (b * Lk) // B if case["ragged"] else Lk for b in range(B)]
    if case["empty"]:
        lens[-1] = 0
    return lens


def _bucket_map(buckets, far, causal):
    """The bucket of each distance key - query from -far to far: one each for the nearest, then in logarithmic steps up to far; with
    causal only distances to keys behind the query matter, otherwise the second half of the buckets is for those ahead. In whole
    numbers: step k starts at the first n with (n / near)^steps >= (far / near)^k."""
    side = buckets if causal else buckets // 2
    near = side // 2
    steps = side - near

    def of(n):
        if n < near:
            return n
        k = 0
        while k + 1 < steps and n ** steps * near ** (k + 1) >= far ** (k + 1) * near ** steps:
            k += 1
        return near + k

    if causal:
        return [of(max(0, -d)) for d in range(-far, far + 1)]
    return [of(abs(d)) + (side if d > 0 else 0) for d in range(-far, far + 1)]


def prepare(case, seed):
    g = _Gen(seed)
    if case["kind"] == "linear8":
        M, N, K = case["M"], case["N"], case["K"]
        wide = -(-K // 128) * 128
        # activations as they leave a normalisation: tokens of different size, a few channels far larger than the others
        x = g.normal((M, K)) * (0.5 + g.uniform((M, 1))) * torch.where(g.uniform((K,)) < 0.01, 12.0, 1.0)
        w = g.normal((N, K), 0.02)
        w_scale = w.abs().amax(1) / 127
        codes = torch.zeros(N, wide, dtype=torch.int8, device=DEV)  # a row's end behind K is zeros
        codes[:, :K] = torch.round(w / w_scale[:, None]).to(torch.int8)
        return {"x": x.to(BF), "w": codes, "w_scale": w_scale, "bias": g.normal((N,), 0.1), **case}
    if case["kind"] == "gated":
        M, F, K = case["M"], case["F"], case["K"]
        s = {"x": g.normal((M, K), dtype=BF), "w": g.normal((2 * F, K), 1.5 / math.sqrt(K), dtype=BF)}  # rows of the gate, then of the other factor
        if case["train"]:
            s["dh"] = g.normal((M, F), 0.1, dtype=BF)
        return {**s, **case}
    B, H, Hk, dh, Lq, Lk = (case[n] for n in ("B", "H", "Hk", "dh", "Lq", "Lk"))
    std = (2.0 / (case["scale"] * math.sqrt(dh))) ** 0.5  # products of a few units whatever the scale
    if Lq == Lk:  # queries, keys and values side by side, as one projection leaves them
        rows = g.normal((B, Lq, (H + 2 * Hk) * dh), std, dtype=BF)
        q, k, v = (t.view(B, Lq, -1, dh) for t in rows.split([H * dh, Hk * dh, Hk * dh], dim=2))
    else:  # a cache with room behind the last key
        room = -(-Lk // 64) * 64 + 64
        q = g.normal((B, Lq, H, dh), std, dtype=BF)
        k, v = (g.normal((B, room, Hk, dh), std, dtype=BF)[:, :Lk] for _ in range(2))
    lens = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV)
    s = {"q": q, "k": k, "v": v, "lens": lens, "first": lens - Lq if case["causal"] and Lq != Lk else None,
         "table": g.normal((case["buckets"], H), 1.0),
         "bucket": torch.tensor(_bucket_map(case["buckets"], case["far"], case["causal"]), dtype=torch.int32, device=DEV)}
    if case["train"]:
        s["do"] = g.normal((B, Lq, H, dh), dtype=BF)
    return {**s, **case}


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _own(s)
    return {"linear8": _plain_linear8, "gated": _plain_gated, "attention": _plain_attention}[s["kind"]](s)


def _own(s):
    from paper_2604_04451_amd import binding as P
    if s["kind"] == "linear8":
        codes, scale = P.chorus_quant_rows_i8(s["x"])
        epilogue = {"bf16": P.EPI_BF16, "gelu": P.EPI_GELU_BF16, "f32": P.EPI_F32}[s["epilogue"]]
        out = torch.empty(s["M"], s["N"], dtype=torch.float32 if s["epilogue"] == "f32" else BF, device=DEV)
        return P.chorus_gemm_i8(codes, scale, s["w"], s["w_scale"], epilogue, out, bias=s["bias"])
    if s["kind"] == "gated":
        act = {"gelu": P.ACT_GELU, "silu": P.ACT_SILU}[s["act"]]
        h = torch.empty(s["M"], s["F"], dtype=BF, device=DEV)
        if not s["train"]:
            return P.chorus_gated_ffn(s["x"], s["w"], act, h)
        pre = torch.empty(s["M"], 2 * s["F"], dtype=BF, device=DEV)
        P.chorus_gated_ffn(s["x"], s["w"], act, h, pre=pre)
        dx, dw = torch.empty_like(s["x"]), torch.empty_like(s["w"])
        P.chorus_gated_ffn_backward(s["x"], s["w"], pre, s["dh"], act, dx, dw)
        return {"h": h, "dx": dx, "dw": dw}
    q, k, v = s["q"], s["k"], s["v"]
    B, Lq, H, dh = q.shape
    o = torch.empty(B, Lq, H, dh, dtype=BF, device=DEV)
    how = {"lens": s["lens"], "first": s["first"], "causal": s["causal"], "scale": s["scale"]}
    if not s["train"]:
        return P.chorus_attention_bias(q, k, v, o, s["table"], s["bucket"], **how)
    lse = torch.empty(B, H, Lq, dtype=torch.float32, device=DEV)
    rest = torch.empty_like(o)
    P.chorus_attention_bias(q, k, v, o, s["table"], s["bucket"], lse=lse, rest=rest, **how)
    dq, dk, dv = (torch.empty(t.shape, dtype=BF, device=DEV) for t in (q, k, v))
    dtable = torch.empty_like(s["table"])
    P.chorus_attention_bias_backward(q, k, v, o, rest, lse, s["do"], s["table"], s["bucket"], dq, dk, dv, dtable, **how)
    return {"o": o, "dq": dq, "dk": dk, "dv": dv, "dtable": dtable}


def _gelu(x):
    return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))


def _plain_linear8(s):
    K = s["K"]
    x = s["x"].float()
    most = x.abs().amax(1)
    codes = torch.round(127.0 * x / torch.where(most > 0, most, 1.0)[:, None])  # 127 x is exact, so that halves are seen
    y = codes @ s["w"][:, :K].float().t() * (most / 127)[:, None] * s["w_scale"] + s["bias"]
    if s["epilogue"] == "gelu":
        y = _gelu(y)
    return y if s["epilogue"] == "f32" else y.to(BF)


def _plain_gated(s):
    F = s["F"]
    x, w = s["x"].float(), s["w"].float()
    g, u = (x @ w.t()).split(F, dim=1)
    if s["act"] == "silu":
        sig = 1.0 / (1.0 + torch.exp(-g))
        a, slope = g * sig, sig * (1.0 + g * (1.0 - sig))
    else:
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (g + 0.044715 * g * g * g))
        a, slope = 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * g * g)
    h = (a * u).to(BF)
    if not s["train"]:
        return h
    dh = s["dh"].float()
    d = torch.cat((dh * u * slope, dh * a), 1)
    return {"h": h, "dx": (d @ w).to(BF), "dw": (d.t() @ x).to(BF)}


def _seen(s, b):
    """[Lq, Lk]: whether the query sees the key, and the distance's place in the bucket map."""
    Lq, Lk = s["Lq"], s["Lk"]
    i, j = torch.arange(Lq, device=DEV)[:, None], torch.arange(Lk, device=DEV)[None]
    at = j - i - (0 if s["first"] is None else s["first"][b])
    see = (j < s["lens"][b]).expand(Lq, Lk)
    return (see & (at <= 0) if s["causal"] else see), at.clamp(-s["far"], s["far"]) + s["far"]


def _plain_attention(s):
    """Sequence by sequence, as many heads at a time as 2 GB of logits hold."""
    q, k, v, train = s["q"], s["k"], s["v"], s["train"]
    B, Lq, H, dh = q.shape
    Hk, Lk, n = k.shape[2], k.shape[1], s["buckets"]
    group = H // Hk
    o = torch.empty(B, Lq, H, dh, dtype=BF, device=DEV)
    if train:
        dq = torch.empty(B, Lq, H, dh, dtype=BF, device=DEV)
        dkv = torch.zeros(2, Hk, Lk, dh, device=DEV)
        dk, dv = (torch.empty(B, Lk, Hk, dh, dtype=BF, device=DEV) for _ in range(2))
        dtable = torch.zeros(n, H, device=DEV)
    step = max(1, min(H, (1 << 29) // (Lq * Lk)))
    for b in range(B):
        see, at = _seen(s, b)
        of = s["bucket"].long()[at]
        if train:
            dkv.zero_()
        for h in range(0, H, step):
            heads = torch.arange(h, min(h + step, H), device=DEV)
            qh = q[b].float().permute(1, 0, 2)[heads]
            kh, vh = (t[b].float().permute(1, 0, 2)[heads // group] for t in (k, v))
            p = torch.bmm(qh, kh.transpose(1, 2).contiguous()).mul_(s["scale"])
            p += s["table"].t()[heads][:, of]
            p.masked_fill_(~see, -math.inf)
            p.sub_(p.amax(2, keepdim=True).clamp(min=torch.finfo(torch.float32).min)).exp_()
            total = p.sum(2, keepdim=True)
            p *= torch.where(total > 0, 1.0 / total, 0.0)
            oh = torch.bmm(p, vh)
            o[b, :, heads] = oh.permute(1, 0, 2).to(BF)
            if not train:
                continue
            do = s["do"][b].float().permute(1, 0, 2)[heads]
            dkv[1].index_add_(0, heads // group, torch.bmm(p.transpose(1, 2).contiguous(), do))
            p *= torch.bmm(do, vh.transpose(1, 2).contiguous()) - (do * oh).sum(2, keepdim=True)
            dq[b, :, heads] = (torch.bmm(p, kh) * s["scale"]).permute(1, 0, 2).to(BF)
            dkv[0].index_add_(0, heads // group, torch.bmm(p.transpose(1, 2).contiguous(), qh) * s["scale"])
            # rows from the last to the first, each one place further to the right than the one before: a column is a distance
            width = Lq + Lk
            skew = torch.zeros(len(heads), Lq, width, device=DEV)
            skew[:, :, :Lk] = p.flip(1)
            by_distance = skew.view(len(heads), -1)[:, :Lq * (width - 1)].view(len(heads), Lq, width - 1).sum(1, dtype=torch.float64)
            place = (torch.arange(width - 1, device=DEV) - (Lq - 1) - (0 if s["first"] is None else s["first"][b])).clamp(-s["far"], s["far"]) + s["far"]
            to = torch.nn.functional.one_hot(s["bucket"].long()[place], n).double()
            dtable[:, heads] += (by_distance @ to).t().float()
        if train:
            dk[b], dv[b] = dkv.permute(0, 2, 1, 3).to(BF)
    return {"o": o, "dq": dq, "dk": dk, "dv": dv, "dtable": dtable} if train else o


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    if case["kind"] == "linear8":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": 2 * M * K + N * K + 8 * N + (4 if case["epilogue"] == "f32" else 2) * M * N, "flops": 2 * M * N * K}
    if case["kind"] == "gated":
        M, F, K, train = case["M"], case["F"], case["K"], case["train"]
        once = 2 * (M * K + 2 * F * K + M * F)
        return {"bytes": once + (once if train else 0), "flops": (12 if train else 4) * M * F * K}
    B, H, Hk, dh, Lq, Lk = (case[n] for n in ("B", "H", "Hk", "dh", "Lq", "Lk"))
    pairs = rows = 0
    for n in _lengths(case):
        rows += n
        if not case["causal"]:
            pairs += Lq * n
            continue
        first = n - Lq if Lq != Lk else 0
        pairs += sum(min(n, max(0, first + i + 1)) for i in range(Lq))
    q, kv = 2 * B * Lq * H * dh, 4 * rows * Hk * dh
    return {"bytes": (4 if case["train"] else 2) * q + (2 if case["train"] else 1) * kv, "flops": (14 if case["train"] else 4) * dh * H * pairs}


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"linear8": _exact_linear8, "gated": _exact_gated, "attention": _exact_attention}[case["kind"]](s)


def _exact_linear8(s):
    """Some rows at a time: scales, codes to the nearest (halves to even), products."""
    M, N, K = s["M"], s["N"], s["K"]
    w = s["w"][:, :K].double().t().contiguous() * s["w_scale"].double()
    y = torch.empty(M, N, dtype=torch.float64, device=DEV)
    for r in range(0, M, 4096):
        x = s["x"][r:r + 4096].double()
        most = x.abs().amax(1, keepdim=True)
        y[r:r + 4096] = torch.nan_to_num(x * 127 / most).round() * (most / 127) @ w
    y += s["bias"].double()
    return _gelu(y) if s["epilogue"] == "gelu" else y


def _exact_gated(s):
    """The gradients by automatic differentiation of the definition."""
    x, w = (s[n].double().requires_grad_(s["train"]) for n in ("x", "w"))
    g, u = x @ w[:s["F"]].t(), x @ w[s["F"]:].t()
    h = (g * torch.sigmoid(g) if s["act"] == "silu" else _gelu(g)) * u
    if not s["train"]:
        return h
    dx, dw = torch.autograd.grad(h, (x, w), s["dh"].double())
    return {"h": h.detach(), "dx": dx, "dw": dw}


def _exact_attention(s):
    """Head by head from the definition, gradients by automatic differentiation; None where the logits of a head are too many."""
    q, k, v, train = s["q"], s["k"], s["v"], s["train"]
    B, Lq, H, dh = q.shape
    group = H // k.shape[2]
    out = {"o": torch.zeros(B, Lq, H, dh, dtype=torch.float64, device=DEV)}
    if train:
        out.update({n: torch.zeros(t.shape, dtype=torch.float64, device=DEV) for n, t in (("dq", q), ("dk", k), ("dv", v), ("dtable", s["table"]))})
    for b in range(B):
        see, at = _seen(s, b)
        place = s["bucket"].long()[at]
        some = see.any(1)[:, None]
        for h in range(H):
            leaves = [t.detach().double().requires_grad_(train) for t in (q[b, :, h], k[b, :, h // group], v[b, :, h // group], s["table"][:, h])]
            one = torch.nn.functional.one_hot(s["bucket"].long(), s["buckets"]).double()  # a distance's bias as a product: no scattered sums behind it
            z = leaves[0] @ leaves[1].t() * s["scale"] + _Pick.apply(one @ leaves[3], at)
            w = torch.softmax(torch.where(some, z.masked_fill(~see, -math.inf), 0.0), 1) * some
            o = w @ leaves[2]
            out["o"][b, :, h] = o.detach()
            if train:
                dq, dk, dv, dt = torch.autograd.grad(o, leaves, s["do"][b, :, h].double())
                out["dq"][b, :, h] = dq
                out["dk"][b, :, h // group] += dk
                out["dv"][b, :, h // group] += dv
                out["dtable"][:, h] += dt
    return out if train else out["o"]


class _Pick(torch.autograd.Function):
    """values[at] for at = clamped distances; the gradient is the sum over each distance's entries."""

    @staticmethod
    def forward(ctx, values, at):
        ctx.save_for_backward(at)
        ctx.n = values.numel()
        return values[at]

    @staticmethod
    def backward(ctx, d):
        (at,) = ctx.saved_tensors
        return torch.bincount(at.reshape(-1), weights=d.reshape(-1), minlength=ctx.n), None
