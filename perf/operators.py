"""Attention over selected blocks of keys and what feeds it, as cases that can be timed and compared.

A video DiT's self-attention runs over tens of thousands of tokens of which a query needs few. A step that uses this rotates its
queries and keys (`rope`), averages them over blocks (`mean`), chooses for every block of 128 queries the key blocks of 64 with the
highest score (`select`) and attends to those only (`attention`).

`own` false: `run` computes the operators from elementary torch operations in 32 bits (angles and scores in 64); true: by the
library's calls. `exact` has the same results in 64 bits, written from the definitions.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
BQ, BK = 128, 64  # queries and keys of a block
LOG2E = 1.4426950408889634


def listed():
    return [
        # 60 tokens of a small edit attend to a 480p clip whose keys and values the program keeps laid out: few rows, a long axis
        _attention("attn_few_60", 12, 12, 128, 60, 32760, 256, kept=True),
        # two frames of a tiny model, shared key heads, three blocks of keys, the last with two: launches and latency
        _attention("attn_tiny_130", 4, 2, 64, 130, 130, 3, scaled=False),
        # a region step of the 1.3B widths: 40 % of a 480p clip, lists of different lengths
        _attention("attn_13104", 12, 12, 128, 13104, 13104, 60, ragged=True),
        # a full 480p step, a fifth of the keys
        _attention("attn_32760", 12, 12, 128, 32760, 32760, 103),
        # the largest: a full 720p step of the 14B widths, a tenth of the keys
        _attention("attn_75600", 40, 40, 128, 75600, 75600, 118),
        # choices for those two steps; the second with text blocks that every query keeps and padding that none may
        _select("select_480p", 12, 12, 128, 256, 512, 103, False),
        _select("select_720p", 40, 40, 128, 591, 1182, 118, True),
        # means of the 480p keys and of the 720p queries
        _mean("mean_480p_keys", 12, 128, 32760, BK),
        _mean("mean_720p_queries", 40, 128, 75600, BQ),
        # an image of 10 x 13 patches: two axes, 40 of a head's 64 values rotated, no normalisation
        _rope("rope_image_130", 4, 64, 130, "none", False, (16, 24), 1.0, 1.0),
        # 480p queries: time, height, width; normalised over the row as the framework's own block does, scaled for attention
        _rope("rope_480p", 12, 128, 32760, "width", False, (44, 42, 42), 1.0, LOG2E / math.sqrt(128)),
        # 720p queries of a model that normalises each head and rotates halves, positions stretched to a larger grid
        _rope("rope_720p", 40, 128, 75600, "head", True, (44, 42, 42), 0.75, 1.0),
    ]


def _attention(name, H, Hk, dh, Lq, Lk, keep, scaled=True, ragged=False, kept=False):
    return {"name": name, "kind": "attention", "H": H, "Hk": Hk, "dh": dh, "Lq": Lq, "Lk": Lk, "keep": keep, "scaled": scaled,
            "ragged": ragged, "kept": kept}


def _select(name, H, Hk, dh, nq, nk, keep, rules):
    return {"name": name, "kind": "select", "H": H, "Hk": Hk, "dh": dh, "nq": nq, "nk": nk, "keep": keep, "rules": rules}


def _mean(name, H, dh, L, block):
    return {"name": name, "kind": "mean", "H": H, "dh": dh, "L": L, "block": block}


def _rope(name, H, dh, L, norm, halves, dims, stretch, scale):
    return {"name": name, "kind": "rope", "H": H, "dh": dh, "L": L, "norm": norm, "halves": halves,
            "dims": " ".join(map(str, dims)), "stretch": stretch, "scale": scale}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "select", "mean", "rope", "rope"])
    dh = rng.choice([64, 128, 128])
    H = rng.choice([1, 4, 5, 8, 12, 12, 16, 40])
    Hk = rng.choice([h for h in (1, 2, 4, H) if H % h == 0]) if rng.random() < 0.3 else H
    if kind == "attention":
        Lk = _log(rng, 64, 75600)
        Lq = Lk if rng.random() < 0.7 else _log(rng, 1, 4096)
        nk = -(-Lk // BK)
        keep = max(1, min(nk, int(nk * math.exp(rng.uniform(math.log(0.05), math.log(0.6))))))
        most = 40 * 75600 * 118
        keep = max(1, min(keep, most // (H * Lq)))
        c = _attention(None, H, Hk, dh, Lq, Lk, keep, rng.random() < 0.6, rng.random() < 0.4, Lq < Lk and rng.random() < 0.5)
    elif kind == "select":
        nk = _log(rng, 1, 2400)
        nq = _log(rng, 1, 600)
        c = _select(None, H, Hk, dh, nq, nk, max(1, int(nk * rng.uniform(0.02, 0.6))), rng.random() < 0.5)
    elif kind == "mean":
        c = _mean(None, H, dh, _log(rng, 1, 75600), rng.choice([BQ, BK]))
    else:
        norm, halves = rng.choice(["none", "width", "head"]), rng.random() < 0.4
        n = rng.randint(1, 4)
        most = dh // n // 2
        dims = [16 * rng.randint(1, max(1, dh // n // 16)) if halves else 2 * rng.randint(max(1, most // 2), most) for _ in range(n)]
        c = _rope(None, H, dh, _log(rng, 1, 75600), norm, halves, dims, rng.choice([1.0, 0.5, rng.uniform(0.4, 2.0)]),
                  rng.choice([1.0, LOG2E / math.sqrt(dh)]))
    c.pop("name")
    return c


# ------------------------------------------------------------------------------------------------ inputs

class _Gen:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(int(seed))

    def normal(self, shape, std=1.0, mean=0.0, dtype=torch.float32):
        t = torch.empty(shape, dtype=torch.float32, device=DEV)
        t.normal_(mean, std, generator=self.g)
        return t.to(dtype)

    def uniform(self, shape):
        return torch.rand(shape, generator=self.g, device=DEV)


def _places(g, H, dh, n, length):
    """[H, n, dh]: what the tokens at n places of a clip have in common, alike where places are near: waves of periods from a
    few blocks of keys to the clip."""
    at = (torch.arange(n, device=DEV) + 0.5) / n * length
    period = 4.0 * torch.exp(g.uniform((H, 1, dh)) * math.log(max(2.0, length / 4)))
    return torch.sin(2 * math.pi * (at[None, :, None] / period + g.uniform((H, 1, dh))))


def _counts(case):
    """How many blocks the list of (head, block of queries) holds."""
    H, nq, keep = case["H"], -(-case["Lq"] // BQ), case["keep"]
    if not case["ragged"]:
        return np.full((H, nq), keep)
    return keep - (np.arange(H)[:, None] * 7 + np.arange(nq)[None] * 3) % (keep // 2 + 1)


def _vt(V, pad):
    """V rows [Lk, D] in the layout that attention reads, [D, pad]: in every 16 tokens position 8c + 4u + i holds 8u + 4c + i."""
    L, D = V.shape
    rows = torch.zeros(pad, D, dtype=V.dtype, device=V.device)
    rows[:L] = V
    return rows.view(pad // 16, 2, 2, 4, D).permute(4, 0, 2, 1, 3).reshape(D, pad).contiguous()


def _prepare_attention(case, g):
    H, Hk, dh, Lq, Lk, keep = (case[n] for n in ("H", "Hk", "dh", "Lq", "Lk", "keep"))
    nq, nk = -(-Lq // BQ), -(-Lk // BK)
    bf = torch.bfloat16
    pad = lambda n: -(-n // 256) * 256  # noqa: E731  as the block pads its tokens
    common = _places(g, Hk, dh, nk, nk)
    blockwise = lambda c, size, L: c.repeat_interleave(size, dim=1)[:, :L]  # noqa: E731
    K = torch.zeros(Hk, pad(Lk), dh, dtype=bf, device=DEV)
    K[:, :Lk] = (blockwise(common, BK, Lk) + g.normal((Hk, Lk, dh), 0.7)).to(bf)
    V = (blockwise(_places(g, Hk, dh, nk, nk), BK, Lk) + g.normal((Hk, Lk, dh), 0.7)).permute(1, 0, 2).reshape(Lk, Hk * dh).to(bf)
    # a block of queries stands where its share of the keys stands; a head adds a little of its own
    at = ((torch.arange(nq, device=DEV) + 0.5) / nq * nk).long().clamp(max=nk - 1)
    asked = common.repeat_interleave(H // Hk, dim=0)[:, at] + g.normal((H, nq, dh), 0.3)
    Q = torch.zeros(H, pad(Lq), dh, dtype=bf, device=DEV)
    Q[:, :Lq] = ((blockwise(asked, BQ, Lq) + g.normal((H, Lq, dh), 0.7)) * (LOG2E / math.sqrt(dh) if case["scaled"] else 1.0)).to(bf)
    score = torch.bmm(asked, common.repeat_interleave(H // Hk, dim=0).transpose(1, 2).contiguous())
    best = torch.topk(score, keep, dim=2).indices
    count = torch.from_numpy(_counts(case)).to(DEV)
    best = torch.where(torch.arange(keep, device=DEV) < count[:, :, None], best, nk).sort(dim=2).values
    blocks = torch.where(best == nk, -1, best).to(torch.int32)
    s = {"Q": Q, "K": K, "V": V, "blocks": blocks}
    if case["kept"]:
        s["Vt"] = _vt(V, pad(Lk))
    return s


def prepare(case, seed):
    g = _Gen(seed)
    bf = torch.bfloat16
    H, dh = case["H"], case["dh"]
    if case["kind"] == "attention":
        return {**_prepare_attention(case, g), **case}
    if case["kind"] == "select":
        Hk, nq, nk = case["Hk"], case["nq"], case["nk"]
        common = _places(g, Hk, dh, nk, nk)
        at = ((torch.arange(nq, device=DEV) + 0.5) / nq * nk).long().clamp(max=nk - 1)
        rule = None
        if case["rules"]:  # the first eighth (at most 8 blocks, a text of 512 tokens) always, the last sixteenth (at most 8) never
            rule = torch.zeros(nk, dtype=torch.uint8, device=DEV)
            rule[:min(8, nk // 8)] = 1
            rule[nk - min(8, nk // 16):] = 2
        return {"Qm": (common.repeat_interleave(H // Hk, dim=0)[:, at] + g.normal((H, nq, dh), 0.3)).to(bf),
                "Km": (common + g.normal((Hk, nk, dh), 0.1)).to(bf), "rule": rule, **case}
    L = case["L"]
    if case["kind"] == "mean":
        pad = -(-L // 256) * 256
        X = torch.zeros(H, pad, dh, dtype=bf, device=DEV)
        n = -(-L // case["block"])
        X[:, :L] = (_places(g, H, dh, n, n).repeat_interleave(case["block"], dim=1)[:, :L] + g.normal((H, L, dh), 0.7)).to(bf)
        return {"X": X, **case}
    # queries, keys and values side by side as a projection leaves them; positions of a grid as near to square as L tokens make
    # it, axis after axis, slowest first
    dims = [int(d) for d in case["dims"].split()]
    n = len(dims)
    side = max(1, int(round(L ** (1.0 / n))))
    i = torch.arange(L, device=DEV)
    places = [(i // side ** (n - 1 - k)) % side if k else i // side ** (n - 1) for k in range(n)]
    freq, axis = [], []
    for k, d in enumerate(dims):
        freq += [10000.0 ** (-2.0 * p / d) for p in range(d // 2)]
        axis += [k] * (d // 2)
    width = H * dh
    return {"x": g.normal((L, 3 * width), 1.5, dtype=bf), "pos": (torch.stack(places, 1) * case["stretch"]).float().contiguous(),
            "freq": torch.tensor(freq, dtype=torch.float64, device=DEV), "axis": torch.tensor(axis, dtype=torch.int32, device=DEV),
            "gain": None if case["norm"] == "none" else g.normal((width if case["norm"] == "width" else dh,), 0.2, 1.3),
            **{**case, "dims": dims}}


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _own(s)
    return {"attention": _plain_attention, "select": _plain_select, "mean": _plain_mean, "rope": _plain_rope}[s["kind"]](s)


def _own(s):
    from paper_2604_04451_amd import binding as B
    bf = torch.bfloat16
    H, dh = s["H"], s["dh"]
    if s["kind"] == "attention":
        Vt = s.get("Vt")
        if Vt is None:
            Vt = torch.empty(s["Hk"] * dh, s["K"].shape[1], dtype=bf, device=DEV)
            B.chorus_v_transpose(s["V"], 0, Vt, s["Lk"])
        O = torch.empty(s["Lq"], H * dh, dtype=bf, device=DEV)
        return B.chorus_attention_blocks(s["Q"], s["K"], Vt, O, s["blocks"], s["Lq"], s["Lk"], prescaled=s["scaled"])
    if s["kind"] == "select":
        blocks = torch.empty(H, s["nq"], s["keep"], dtype=torch.int32, device=DEV)
        return B.chorus_block_select(s["Qm"], s["Km"], blocks, rule=s["rule"])
    if s["kind"] == "mean":
        out = torch.empty(H, -(-s["L"] // s["block"]), dh, dtype=bf, device=DEV)
        return B.chorus_block_mean(s["X"], out, s["L"], s["block"])
    out = torch.empty(H, -(-s["L"] // 256) * 256, dh, dtype=bf, device=DEV)
    norm = {"none": B.ROPE_NORM_NONE, "width": B.ROPE_NORM_WIDTH, "head": B.ROPE_NORM_HEAD}[s["norm"]]
    return B.chorus_rope_axes(s["x"], 0, s["gain"], norm, out, s["L"], H, dh, s["pos"], s["freq"], s["axis"],
                              layout=B.ROPE_HALVES if s["halves"] else B.ROPE_PAIRS, out_scale=s["scale"])


def _plain_attention(s):
    """The listed blocks gathered, some lists at a time (all together they are larger than the card), one softmax over each."""
    Q, K, V, blocks = s["Q"], s["K"], s["V"], s["blocks"]
    H, Hk, dh, Lq, Lk = s["H"], s["Hk"], s["dh"], s["Lq"], s["Lk"]
    _, nq, keep = blocks.shape
    n = K.shape[1] // BK
    Kb = K.reshape(Hk * n, BK, dh)
    Vb = torch.nn.functional.pad(V, (0, 0, 0, n * BK - Lk)).view(n, BK, Hk, dh).permute(2, 0, 1, 3).reshape(Hk * n, BK, dh)
    Qb = torch.nn.functional.pad(Q[:, :Lq], (0, 0, 0, nq * BQ - Lq)).view(H * nq, BQ, dh)
    lists = blocks.view(H * nq, keep).long()
    first = torch.arange(H * nq, device=Q.device) // nq // (H // Hk) * n
    at = first[:, None] + lists.clamp(min=0)
    key = lists[:, :, None] * BK + torch.arange(BK, device=Q.device)
    out_of = ((lists < 0)[:, :, None] | (key >= Lk)).view(H * nq, 1, keep * BK)
    O = torch.empty(H * nq, BQ, dh, dtype=torch.bfloat16, device=Q.device)
    step = max(1, (1 << 29) // (keep * BK * dh))
    for a in range(0, H * nq, step):
        of = slice(a, a + step)
        k = Kb[at[of]].float().view(-1, keep * BK, dh)
        p = torch.bmm(Qb[of].float(), k.transpose(1, 2).contiguous())
        if not s["scaled"]:
            p *= LOG2E / math.sqrt(dh)
        p.masked_fill_(out_of[of], -math.inf)
        p.sub_(p.amax(2, keepdim=True).clamp(min=torch.finfo(torch.float32).min)).exp2_()
        o = torch.bmm(p, Vb[at[of]].float().view(-1, keep * BK, dh))
        total = p.sum(2, keepdim=True)
        O[of] = torch.where(total > 0, o / total, 0.0).to(torch.bfloat16)
    return O.view(H, nq * BQ, dh)[:, :Lq].permute(1, 0, 2).reshape(Lq, H * dh)


def _plain_select(s):
    """Scores in 64 bits: neighbours in rank are as near as 32 bits round."""
    nk, keep = s["nk"], s["keep"]
    score = torch.matmul(s["Qm"].double(), s["Km"].double().transpose(1, 2).contiguous().repeat_interleave(s["H"] // s["Hk"], dim=0))
    order = torch.sort(score, dim=2, descending=True, stable=True).indices
    if s["rule"] is not None:
        rank = torch.tensor([1, 0, 2], device=order.device)[s["rule"].long()]  # always, by score, never
        order = torch.gather(order, 2, torch.sort(rank[order], dim=2, stable=True).indices)
        order = torch.where(rank[order] == 2, nk, order)
    return _ascending(order[:, :, :keep], nk)


def _ascending(chosen, nk):
    chosen = chosen.sort(dim=2).values
    return torch.where(chosen == nk, -1, chosen).to(torch.int32)


def _plain_mean(s):
    X, L, block = s["X"], s["L"], s["block"]
    n = -(-L // block)
    rows = torch.nn.functional.pad(X[:, :L].float(), (0, 0, 0, n * block - L)).view(X.shape[0], n, block, X.shape[2])
    count = (L - torch.arange(n, device=X.device) * block).clamp(max=block)
    return (rows.sum(2) / count[:, None]).to(torch.bfloat16)


def _plain_rope(s):
    L, H, dh = s["L"], s["H"], s["dh"]
    x = s["x"][:, :H * dh].float()
    if s["norm"] == "width":
        x = x * torch.rsqrt((x * x).mean(1, keepdim=True) + 1e-6) * s["gain"]
    x = x.view(L, H, dh)
    if s["norm"] == "head":
        x = x * torch.rsqrt((x * x).mean(2, keepdim=True) + 1e-6) * s["gain"]
    n = s["freq"].numel()
    angle = s["pos"].double()[:, s["axis"].long()] * s["freq"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if s["halves"]:
        a, b = x[:, :, :n], x[:, :, n:2 * n]
        y = torch.cat((a * cos - b * sin, a * sin + b * cos, x[:, :, 2 * n:]), 2)
    else:
        a, b = x[:, :, 0:2 * n:2], x[:, :, 1:2 * n:2]
        y = torch.cat((torch.stack((a * cos - b * sin, a * sin + b * cos), 3).flatten(2), x[:, :, 2 * n:]), 2)
    out = torch.zeros(H, -(-L // 256) * 256, dh, dtype=torch.bfloat16, device=x.device)
    out[:, :L] = (y * s["scale"]).to(torch.bfloat16).permute(1, 0, 2)
    return out


# ------------------------------------------------------------------------------------------------ what a pass cannot do without

def work(case):
    H, dh = case["H"], case["dh"]
    if case["kind"] == "attention":
        Lq, Lk = case["Lq"], case["Lk"]
        counts = _counts(case)
        rows = np.minimum(BQ, Lq - np.arange(counts.shape[1]) * BQ)
        keys = np.minimum(counts * BK, Lk)
        used = min(1.0, counts.sum() / case["Hk"] / (-(-Lk // BK)))  # keys and values: each once, those that some list can hold
        return {"bytes": 4 * Lq * H * dh + int(4 * Lk * case["Hk"] * dh * used) + 4 * int(counts.sum()),
                "flops": 4 * dh * int((rows[None] * keys).sum())}
    if case["kind"] == "select":
        nq, nk = case["nq"], case["nk"]
        return {"bytes": 2 * dh * (H * nq + case["Hk"] * nk) + 4 * H * nq * case["keep"] + nk * case["rules"], "flops": 2 * H * nq * nk * dh}
    L = case["L"]
    if case["kind"] == "mean":
        return {"bytes": 2 * H * dh * (L - (-L // case["block"])), "flops": H * dh * L}
    n = len(case["dims"].split())
    return {"bytes": 2 * H * dh * (L + -(-L // 256) * 256) + 4 * n * L, "flops": 10 * H * dh * L}


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "select": _exact_select, "mean": _exact_mean, "rope": _exact_rope}[case["kind"]](s)


def _exact_attention(s):
    """Every logit of some rows of one head, those of keys outside the row's list taken out."""
    H, Hk, dh, Lq, Lk = s["H"], s["Hk"], s["dh"], s["Lq"], s["Lk"]
    nk = -(-Lk // BK)
    out = torch.zeros(Lq, H, dh, dtype=torch.float64, device=DEV)
    rows = BQ * max(1, (1 << 26) // Lk // BQ)
    for h in range(H):
        k = s["K"][h // (H // Hk), :Lk].double()
        v = s["V"].view(Lk, Hk, dh)[:, h // (H // Hk)].double()
        listed_by = torch.zeros(s["blocks"].shape[1], nk + 1, dtype=torch.bool, device=DEV)
        listed_by.scatter_(1, torch.where(s["blocks"][h] < 0, nk, s["blocks"][h]).long(), True)
        for r in range(0, Lq, rows):
            q = s["Q"][h, r:min(r + rows, Lq)].double()
            z = q @ k.t().contiguous() * (math.log(2.0) if s["scaled"] else 1 / math.sqrt(dh))
            block = torch.arange(r, r + q.shape[0], device=DEV) // BQ
            off = ~listed_by[block, :nk].repeat_interleave(BK, dim=1)[:, :Lk]
            z.masked_fill_(off, -math.inf)
            w = torch.nan_to_num(torch.exp(z - z.max(1, keepdim=True).values), nan=0.0)
            total = w.sum(1, keepdim=True)
            out[r:r + rows, h] = torch.where(total > 0, (w @ v) / total, torch.zeros_like(total))
    return out.view(Lq, H * dh)


def _exact_select(s):
    """On the host: block by block of queries, by (class, score, index)."""
    Qm, Km = s["Qm"].double().cpu().numpy(), s["Km"].double().cpu().numpy()
    H, Hk, nq, nk, keep = s["H"], s["Hk"], s["nq"], s["nk"], s["keep"]
    rule = np.zeros(nk, np.int64) if s["rule"] is None else s["rule"].cpu().numpy().astype(np.int64)
    forced, free = np.flatnonzero(rule == 1), np.flatnonzero(rule == 0)
    out = np.full((H, nq, keep), -1, np.int32)
    for h in range(H):
        score = Qm[h] @ Km[h // (H // Hk)].T
        by = [of[np.argsort(-score[:, of], axis=1, kind="stable")] for of in (forced, free)]
        chosen = np.concatenate(by, axis=1)[:, :keep]
        out[h, :, :chosen.shape[1]] = np.sort(chosen, axis=1)
    return torch.from_numpy(out).to(DEV)


def _exact_mean(s):
    X, L, block = s["X"], s["L"], s["block"]
    whole = L // block
    parts = [X[:, :whole * block].double().view(X.shape[0], whole, block, X.shape[2]).mean(2)]
    if L % block:
        parts.append(X[:, whole * block:L].double().mean(1, keepdim=True))
    return torch.cat(parts, 1)


def _exact_rope(s):
    """Pairs as complex numbers, turned by exp(i angle)."""
    L, H, dh = s["L"], s["H"], s["dh"]
    n = s["freq"].numel()
    turn = torch.polar(torch.ones(L, n, dtype=torch.float64, device=DEV), s["pos"].double()[:, s["axis"].long()] * s["freq"])
    out = torch.zeros(H, -(-L // 256) * 256, dh, dtype=torch.float64, device=DEV)
    rstd = None
    if s["norm"] == "width":
        rstd = (s["x"][:, :H * dh].double().pow(2).mean(1) + 1e-6).rsqrt()
    for h in range(H):
        x = s["x"][:, h * dh:(h + 1) * dh].double()
        if s["norm"] == "width":
            x = x * rstd[:, None] * s["gain"][h * dh:(h + 1) * dh].double()
        elif s["norm"] == "head":
            x = x * (x.pow(2).mean(1, keepdim=True) + 1e-6).rsqrt() * s["gain"].double()
        one, two = (slice(0, n), slice(n, 2 * n)) if s["halves"] else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
        z = torch.complex(x[:, one].contiguous(), x[:, two].contiguous()) * turn
        x = x.clone()
        x[:, one], x[:, two] = z.real, z.imag
        out[h, :L] = x * s["scale"]
    return out
