"""The operators of attention whose speed is measured, as a training or serving program calls them.

Between a stage's first product (queries, keys and values at once) and its second one, a layer normalises and rotates
its heads and attends: to a whole prompt in training and where a prompt is taken in, to a paged cache where tokens are
made one at a time.  One case is one call on tensors the program holds: `prepare` makes them, `run` computes.

  heads          root-mean-square norm of each query's and key's head, and its rotation by the token's position; with a
                 cache, keys and values go to their slots there in the same pass
  heads_grad     its gradients: of queries and keys, and of the norms' weights summed over tokens and heads
  prompt         causal attention of packed sequences with grouped heads, with the statistics the backward pass keeps
  prompt_grad    its gradients
  token          attention of one new token of each sequence over a paged cache
"""

import math
import random

import torch

own = False

BYTES = {"float16": 2, "bfloat16": 2, "float32": 4}
EPS = 1e-6
BASE = 10000.0


def listed():
    return [
        # one decode step of a 64-sequence batch, 5120 wide, keys and values into the cache: latency
        dict(name="heads_decode64_fp16", op="heads", dtype="float16", weights="float16", tokens=64, heads=40,
             kv_heads=40, dim=128, rotary=128, interleaved=False, first=1000, page=16, pool=1031),
        # GPT-3-width queries and keys of 8 sequences of 2048: the largest
        dict(name="heads_gpt3_bf16", op="heads", dtype="bfloat16", weights="float32", tokens=16384, heads=96,
             kv_heads=96, dim=128, rotary=128, interleaved=False, first=0, page=0, pool=0),
        # a next-token sequence (2047), grouped heads of 80, half of each rotated, neighbours paired
        dict(name="heads_grad_ragged_fp16", op="heads_grad", dtype="float16", weights="float32", tokens=2047, heads=40,
             kv_heads=10, dim=80, rotary=40, interleaved=True, first=131072, page=0, pool=0),
        # backward of the GPT layer, 8 x 1024 tokens of 4096
        dict(name="heads_grad_gpt_bf16", op="heads_grad", dtype="bfloat16", weights="bfloat16", tokens=8192, heads=32,
             kv_heads=32, dim=128, rotary=128, interleaved=False, first=0, page=0, pool=0),
        # a few short prompts, one of a single token: latency
        dict(name="prompt_short_fp16", op="prompt", dtype="float16", heads=40, kv_heads=8, dim=128, sequences=8,
             longest=61, before=0),
        # prompts of all lengths packed together, the last part of each after a prefix that the cache had
        dict(name="prompt_packed_bf16", op="prompt", dtype="bfloat16", heads=32, kv_heads=8, dim=128, sequences=24,
             longest=4095, before=512),
        # one long document: the largest
        dict(name="prompt_long_bf16", op="prompt", dtype="bfloat16", heads=32, kv_heads=8, dim=128, sequences=1,
             longest=16384, before=0),
        # backward of packed next-token sequences, heads of 64
        dict(name="prompt_grad_ragged_fp16", op="prompt_grad", dtype="float16", heads=40, kv_heads=8, dim=64,
             sequences=13, longest=2047, before=0),
        # backward of the GPT-3-width layer, 8 sequences of 2048 tokens
        dict(name="prompt_grad_gpt3_bf16", op="prompt_grad", dtype="bfloat16", heads=96, kv_heads=96, dim=128,
             sequences=8, longest=2048, before=0, even=True),
        # one sequence being answered: latency
        dict(name="token_one_bf16", op="token", dtype="bfloat16", heads=32, kv_heads=8, dim=128, sequences=1,
             longest=2047, page=16),
        # a decode step of 64 sequences of all lengths, as many key heads as query heads
        dict(name="token_decode64_fp16", op="token", dtype="float16", heads=40, kv_heads=40, dim=128, sequences=64,
             longest=4096, page=16),
        # a few very long contexts, grouped heads, a page length that no tile divides
        dict(name="token_long_bf16", op="token", dtype="bfloat16", heads=32, kv_heads=8, dim=128, sequences=6,
             longest=131000, page=48, even=True),
    ]


# ------------------------------------------------------------------ the ranges

def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["heads", "heads_grad", "prompt", "prompt", "prompt_grad", "token", "token"])
    while True:
        kv = rng.choice([1, 2, 3, 4, 8, 10, 16, 32, 40])
        case = dict(op=op, dtype=rng.choice(["float16", "bfloat16"]), heads=kv * rng.choice([1, 1, 2, 4, 5, 8]),
                    kv_heads=kv, dim=rng.choice([64, 128, 128, 8 * rng.randint(2, 16)]))
        if case["heads"] > 128:
            continue
        if op in ("heads", "heads_grad"):
            case["dtype"] = rng.choice([case["dtype"], case["dtype"], "float32"])
            cached = op == "heads" and rng.random() < 0.5
            page = rng.choice([1, 16, 24, 64, 256])
            case.update(weights=rng.choice([case["dtype"], "float32"]), tokens=_log(rng, 1, 2048 if cached else 16384),
                        interleaved=rng.random() < 0.5, first=_log(rng, 1, 1 << 20))
            case.update(rotary=rng.choice([case["dim"], case["dim"] // 4 * 2]), page=page if cached else 0,
                        pool=case["tokens"] // page + rng.randint(1, 64) if cached else 0)
            if work(case)["bytes"] <= 1.6e9:
                return case
        elif op == "token":
            case.update(sequences=_log(rng, 1, 256), longest=_log(rng, 1, 131072), page=rng.choice([1, 16, 24, 64, 256]),
                        even=rng.random() < 0.3)
            if work(case)["bytes"] <= 3.2e9:
                return case
        else:
            case.update(sequences=_log(rng, 1, 64), longest=_log(rng, 1, 16384), before=rng.choice([0, _log(rng, 1, 4096)]),
                        even=rng.random() < 0.3)
            if op == "prompt_grad":
                case["before"] = 0
            if work(case)["flops"] <= (2.19e12 if op == "prompt" else 2.06e12) and max(_lengths(case)) ** 2 <= 2.7e8:
                return case


def _lengths(case):
    """The sequences' lengths: one the longest, the others of all sizes, the same for every seed."""
    n, longest = case["sequences"], case["longest"]
    if case.get("even"):
        return [longest] * n
    rng = random.Random(f"{n} {longest} {case['heads']} {case['dim']}")
    out = [_log(rng, 1, longest) for _ in range(n)]
    out[rng.randrange(n)] = longest
    return out


def _before(case):
    """Keys that a sequence has before its first query."""
    rng = random.Random(f"{case['before']} {case['sequences']}")
    return [rng.randint(0, case["before"]) for _ in range(case["sequences"])]


# ------------------------------------------------------------------ inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _projected(g, tokens, heads, dim, dtype):
    """What a product gives: of another size from head to head, one channel in 64 wide."""
    wide = torch.where(torch.rand(heads, dim, generator=g, device="cuda") < 1 / 64, 6.0, 1.0)
    size = torch.exp(0.5 * _randn(g, heads, 1))
    return _randn(g, tokens, heads, dim).mul_(wide * size).to(getattr(torch, dtype))


def _gradient(g, tokens, heads, dim, dtype):
    """Small, and of another size from token to token."""
    return _randn(g, tokens, heads, dim).mul_(1e-2 * torch.exp(_randn(g, tokens, 1, 1))).to(getattr(torch, dtype))


def _offsets(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _frequencies(case):
    half = case["rotary"] // 2
    return BASE ** (-torch.arange(half, dtype=torch.float64, device="cuda") / max(half, 1))


def prepare(case, seed):
    g, op, dim, dtype = _generator(seed), case["op"], case["dim"], case["dtype"]
    heads, kv = case["heads"], case["kv_heads"]
    s = {"op": op, "case": case, "scale": dim ** -0.5}
    if op in ("heads", "heads_grad"):
        t, wt = case["tokens"], getattr(torch, case["weights"])
        # queries, keys and values of a token beside each other, as one product leaves them
        qkv = _projected(g, t, heads + 2 * kv, dim, dtype)
        s["q"], s["k"], s["v"] = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
        s["wq"], s["wk"] = ((1 + 0.1 * _randn(g, dim)).to(wt) for _ in range(2))
        s["frequencies"] = _frequencies(case)
        s["positions"] = torch.randint(0, 64, (t,), generator=g, device="cuda", dtype=torch.int32) + case["first"]
        if op == "heads_grad":
            s["dq"], s["dk"] = _gradient(g, t, heads, dim, dtype), _gradient(g, t, kv, dim, dtype)
        if case["page"]:
            shape = case["pool"], case["page"], kv, dim
            s["k_cache"], s["v_cache"] = (_randn(g, *shape).to(getattr(torch, dtype)) for _ in range(2))
            s["slots"] = torch.randperm(case["pool"] * case["page"], generator=g, device="cuda")[:t].int()
        return s
    lengths = _lengths(case)
    if op == "token":
        n, page = len(lengths), case["page"]
        need = [-(-length // page) for length in lengths]
        pool = sum(need) + 5  # some pages of the pool are nobody's
        order = torch.randperm(pool, generator=g, device="cuda").int()
        table = torch.zeros(n, max(need), dtype=torch.int32, device="cuda")
        for i, at in enumerate(_offsets(need)[:-1]):
            table[i, :need[i]] = order[at:at + need[i]]
        t = getattr(torch, dtype)
        s["q"] = _randn(g, n, heads, dim).to(t)
        s["k_cache"], s["v_cache"] = (torch.empty(pool, page, kv, dim, dtype=t, device="cuda").normal_(generator=g)
                                      for _ in range(2))
        s.update(pages=table, lengths=_int32(lengths), on_host=lengths)
        return s
    before = _before(case)
    q_at, k_at = _offsets(lengths), _offsets([a + b for a, b in zip(lengths, before)])
    s["q"] = _projected(g, q_at[-1], heads, dim, dtype)
    s["k"], s["v"] = (_projected(g, k_at[-1], kv, dim, dtype) for _ in range(2))
    s.update(q_offsets=_int32(q_at), k_offsets=_int32(k_at), on_host=(q_at, k_at))
    if op == "prompt_grad":
        s["dout"] = _gradient(g, q_at[-1], heads, dim, dtype)
        out, s["lse"] = _prompt_plain(s)
        s["out"] = out.to(s["q"].dtype)
    return s


# ------------------------------------------------------------------ run

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2211_05322_amd import binding as B

    op = s["op"]
    if op == "heads":
        pair = s["case"]["interleaved"]
        if "slots" in s:
            q, _ = B.reshard_rotate_heads(s["q"], s["k"], s["wq"], s["wk"], EPS, s["frequencies"], s["positions"], pair,
                                          v=s["v"], cache=(s["k_cache"], s["v_cache"]), slots=s["slots"])
            return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
        q, k = B.reshard_rotate_heads(s["q"], s["k"], s["wq"], s["wk"], EPS, s["frequencies"], s["positions"], pair)
        return {"q": q, "k": k}
    if op == "heads_grad":
        dq, dk, dwq, dwk = B.reshard_rotate_heads_backward(
            s["dq"], s["dk"], s["q"], s["k"], s["wq"], s["wk"], EPS, s["frequencies"], s["positions"],
            s["case"]["interleaved"])
        return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}
    if op == "prompt":
        out, lse = B.reshard_attention(s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"], scale=s["scale"])
        return {"out": out, "lse": lse}
    if op == "prompt_grad":
        dq, dk, dv = B.reshard_attention_backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"],
                                                  s["q_offsets"], s["k_offsets"], scale=s["scale"])
        return {"dq": dq, "dk": dk, "dv": dv}
    return B.reshard_attention_paged(s["q"], s["k_cache"], s["v_cache"], s["pages"], s["lengths"], scale=s["scale"])


def _pairs(x, rotary, interleaved):
    """The rotated part of each head as two tensors of its pairs' first and second elements, and the rest."""
    part, rest = x[..., :rotary], x[..., rotary:]
    if interleaved:
        return part[..., 0::2], part[..., 1::2], rest
    return part[..., :rotary // 2], part[..., rotary // 2:], rest


def _joined(a, b, rest, interleaved):
    part = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((part, rest), -1)


def _turned(x, s, way):
    """Heads rotated by their token's angles; way = -1 turns them back."""
    angle = s["positions"].double()[:, None, None] * s["frequencies"]  # far positions lose their angle in 32 bits
    c, n = angle.cos().to(x.dtype), way * angle.sin().to(x.dtype)
    a, b, rest = _pairs(x, s["case"]["rotary"], s["case"]["interleaved"])
    return _joined(a * c - b * n, b * c + a * n, rest, s["case"]["interleaved"])


def _heads_plain(x, w, s):
    x = x.float()
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)
    return _turned(x * r * w.float(), s, 1)


def _heads_grad_plain(dy, x, w, s):
    x = x.float()
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)
    g, xhat = _turned(dy.float(), s, -1), x * r
    dw = (g * xhat).sum((0, 1))
    g = g * w.float()
    return r * (g - xhat * (g * xhat).mean(-1, keepdim=True)), dw


def _visible(lq, lk):
    """Whether query i sees key j: the last query sees all."""
    i = torch.arange(lq, device="cuda")[:, None]
    return torch.arange(lk, device="cuda")[None, :] <= i + (lk - lq)


def _parts(s, each=1 << 30):
    """(query rows, key rows, key head) of the sequences, a key head and a stretch of its queries at a time."""
    q_at, k_at = s["on_host"]
    group = s["q"].shape[1] // s["k"].shape[1]
    for q0, q1, k0, k1 in zip(q_at, q_at[1:], k_at, k_at[1:]):
        lq, lk = q1 - q0, k1 - k0
        step = max(1, each // (4 * group * max(lk, 1)))  # rows whose scores fit
        heads = max(1, min(s["k"].shape[1], each // (4 * group * max(lq * lk, 1))))
        for h in range(0, s["k"].shape[1], heads):
            for lo in range(0, lq, step):
                yield q0, lq, k0, lk, lo, min(lq, lo + step), h, min(s["k"].shape[1], h + heads), group


def _scores(s, q, k, lq, lk, lo, hi):
    x = torch.matmul(q, k.transpose(1, 2).contiguous()) * s["scale"]
    return x.masked_fill(~_visible(lq, lk)[lo:hi].repeat(q.shape[1] // (hi - lo), 1), -math.inf)


def _by_key_head(x, a, b, heads_from, heads_to, group):
    """Rows a to b of heads that share a key head, one after the other: [key heads, group * rows, dim]."""
    x = x[a:b, heads_from * group:heads_to * group].float()
    return x.unflatten(1, (heads_to - heads_from, group)).permute(1, 2, 0, 3).flatten(1, 2).contiguous()


def _back(x, group):
    """[rows, heads, dim] of the form above."""
    return x.unflatten(1, (group, -1)).permute(2, 0, 1, 3).flatten(1, 2)


def _prompt_plain(s):
    out = torch.empty(s["q"].shape, device="cuda")
    lse = torch.empty(s["q"].shape[1], s["q"].shape[0], device="cuda")
    for q0, lq, k0, lk, lo, hi, h0, h1, group in _parts(s):
        q = _by_key_head(s["q"], q0 + lo, q0 + hi, h0, h1, group)
        k, v = (_by_key_head(s[name], k0, k0 + lk, h0, h1, 1) for name in "kv")
        x = _scores(s, q, k, lq, lk, lo, hi)
        top = x.amax(-1, keepdim=True)
        p = torch.exp(x - top)
        total = p.sum(-1, keepdim=True)
        out[q0 + lo:q0 + hi, h0 * group:h1 * group] = _back(torch.matmul(p, v) / total, group)
        lse[h0 * group:h1 * group, q0 + lo:q0 + hi] = (top + total.log()).view((h1 - h0) * group, hi - lo)
    return out, lse


def _prompt_grad_plain(s):
    dq, dk, dv = (torch.zeros(s[name].shape, device="cuda") for name in "qkv")
    for q0, lq, k0, lk, lo, hi, h0, h1, group in _parts(s):
        q, dout, out = (_by_key_head(s[name], q0 + lo, q0 + hi, h0, h1, group) for name in ("q", "dout", "out"))
        k, v = (_by_key_head(s[name], k0, k0 + lk, h0, h1, 1) for name in "kv")
        lse = s["lse"][h0 * group:h1 * group, q0 + lo:q0 + hi].reshape(h1 - h0, -1, 1)
        p = torch.exp(_scores(s, q, k, lq, lk, lo, hi) - lse)
        dp = torch.matmul(dout, v.transpose(1, 2).contiguous())
        ds = p * (dp - (dout * out).sum(-1, keepdim=True)) * s["scale"]
        dq[q0 + lo:q0 + hi, h0 * group:h1 * group] = _back(torch.matmul(ds, k), group)
        dk[k0:k0 + lk, h0:h1] += _back(torch.matmul(ds.transpose(1, 2).contiguous(), q), 1)
        dv[k0:k0 + lk, h0:h1] += _back(torch.matmul(p.transpose(1, 2).contiguous(), dout), 1)
    return dq, dk, dv


def _token_plain(s):
    n, heads, dim = s["q"].shape
    kv = s["k_cache"].shape[2]
    out = torch.empty(n, heads, dim, device="cuda")
    for i, length in enumerate(s["on_host"]):
        pages = s["pages"][i, :-(-length // s["case"]["page"])].long()
        k, v = (s[name][pages].flatten(0, 1)[:length].float().transpose(0, 1).contiguous()
                for name in ("k_cache", "v_cache"))
        x = torch.matmul(s["q"][i].float().view(kv, heads // kv, dim), k.transpose(1, 2).contiguous()) * s["scale"]
        p = torch.exp(x - x.amax(-1, keepdim=True))
        out[i] = (torch.matmul(p, v) / p.sum(-1, keepdim=True)).view(heads, dim)
    return out


def _run_plain(s):
    op, t = s["op"], s["q"].dtype
    if op == "heads":
        q, k = _heads_plain(s["q"], s["wq"], s).to(t), _heads_plain(s["k"], s["wk"], s).to(t)
        if "slots" not in s:
            return {"q": q, "k": k}
        at = s["slots"].long()
        s["k_cache"].flatten(0, 1)[at] = k
        s["v_cache"].flatten(0, 1)[at] = s["v"]
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if op == "heads_grad":
        dq, dwq = _heads_grad_plain(s["dq"], s["q"], s["wq"], s)
        dk, dwk = _heads_grad_plain(s["dk"], s["k"], s["wk"], s)
        return {"dq": dq.to(t), "dk": dk.to(t), "dwq": dwq, "dwk": dwk}
    if op == "prompt":
        out, lse = _prompt_plain(s)
        return {"out": out.to(t), "lse": lse}
    if op == "prompt_grad":
        dq, dk, dv = _prompt_grad_plain(s)
        return {"dq": dq.to(t), "dk": dk.to(t), "dv": dv.to(t)}
    return _token_plain(s).to(t)


# ------------------------------------------------------------------ work

def _seen(case):
    """Pairs of a query and a key that it sees, of one head."""
    return sum(n * b + n * (n + 1) // 2 for n, b in zip(_lengths(case), _before(case)))


def work(case):
    op, e, d, h, kv = case["op"], BYTES[case["dtype"]], case["dim"], case["heads"], case["kv_heads"]
    if op in ("heads", "heads_grad"):
        t, w = case["tokens"], 2 * d * BYTES[case["weights"]] + 4 * case["rotary"]
        if op == "heads":
            values = 2 * kv * d * e if case["page"] else 0  # read and written
            return {"bytes": t * (2 * (h + kv) * d * e + values + 4 + (4 if case["page"] else 0)) + w,
                    "flops": 8 * t * (h + kv) * d}
        return {"bytes": t * (3 * (h + kv) * d * e + 4) + w + 8 * d, "flops": 16 * t * (h + kv) * d}
    if op == "token":
        n, tokens = case["sequences"], sum(_lengths(case))
        return {"bytes": 2 * tokens * kv * d * e + 2 * n * h * d * e + 4 * (n + tokens // case["page"]),
                "flops": 4 * tokens * h * d}
    nq, nk = sum(_lengths(case)), sum(_lengths(case)) + sum(_before(case))
    if op == "prompt":
        return {"bytes": 2 * nq * h * d * e + 2 * nk * kv * d * e + 4 * nq * h, "flops": 4 * _seen(case) * h * d}
    return {"bytes": 4 * nq * h * d * e + 4 * nk * kv * d * e + 4 * nq * h, "flops": 10 * _seen(case) * h * d}


# ------------------------------------------------------------------ the definition in 64 bits

def _rotation_64(s, tokens):
    """Each token's rotation as a matrix [tokens, dim, dim] that acts on a head from the left, without its zeros: the
    cosine at every element, and the sine with its sign at the element that each takes its partner from."""
    d, r = s["case"]["dim"], s["case"]["rotary"]
    cos = torch.ones(tokens, d, dtype=torch.float64, device="cuda")
    sin, partner = torch.zeros_like(cos), torch.arange(d, device="cuda")
    for j in range(r // 2):
        i0, i1 = (2 * j, 2 * j + 1) if s["case"]["interleaved"] else (j, j + r // 2)
        angle = s["positions"].double() * BASE ** (-j / (r // 2))
        cos[:, i0] = cos[:, i1] = torch.cos(angle)
        sin[:, i0], sin[:, i1] = -torch.sin(angle), torch.sin(angle)
        partner[i0], partner[i1] = i1, i0
    return cos[:, None], sin[:, None], partner


def _heads_64(x, w, turn):
    x = x.double()
    y = x * (torch.linalg.vecdot(x, x)[..., None] / x.shape[-1] + EPS) ** -0.5 * w.double()
    cos, sin, partner = turn
    return cos * y + sin * y[..., partner]


def _heads_grad_64(dy, x, w, turn):
    dy, x, w = dy.double(), x.double(), w.double()
    cos, sin, partner = turn
    g = cos * dy + (sin * dy)[..., partner]  # the transposed rotation
    r = (torch.linalg.vecdot(x, x)[..., None] / x.shape[-1] + EPS) ** -0.5
    # y = x r w with r = (x.x / d + eps)^(-1/2):  dx = r w g - x r^3 (x . w g) / d
    dx = r * w * g - x * r ** 3 * torch.linalg.vecdot(x, w * g)[..., None] / x.shape[-1]
    return dx, torch.linalg.vecdot((x * r).flatten(0, 1), g.flatten(0, 1), dim=0)


def _weights_64(s, i, head, group, lo, hi):
    """(attention weights, logarithm of their sum) of rows lo to hi of sequence i in one head."""
    q_at, k_at = s["on_host"]
    lq, lk = q_at[i + 1] - q_at[i], k_at[i + 1] - k_at[i]
    k = s["k"][k_at[i]:k_at[i + 1], head // group].double()
    x = s["scale"] * (s["q"][q_at[i] + lo:q_at[i] + hi, head].double() @ k.t())
    x = x.tril(lk - lq + lo) + torch.full_like(x, -math.inf).triu(lk - lq + lo + 1)
    lse = torch.logsumexp(x, 1)
    return x, lse


def exact(case, seed):
    s = prepare(case, seed)
    op = s["op"]
    if op in ("heads", "heads_grad"):
        turn = _rotation_64(s, case["tokens"])
        if op == "heads_grad":
            dq, dwq = _heads_grad_64(s["dq"], s["q"], s["wq"], turn)
            dk, dwk = _heads_grad_64(s["dk"], s["k"], s["wk"], turn)
            return {"dq": dq, "dk": dk, "dwq": dwq, "dwk": dwk}
        q, k = _heads_64(s["q"], s["wq"], turn), _heads_64(s["k"], s["wk"], turn)
        if not case["page"]:
            return {"q": q, "k": k}
        caches = s["k_cache"].double(), s["v_cache"].double()
        for cache, rows in zip(caches, (k, s["v"].double())):
            cache.view(-1, case["kv_heads"], case["dim"]).index_copy_(0, s["slots"].long(), rows)
        return {"q": q, "k_cache": caches[0], "v_cache": caches[1]}
    group = case["heads"] // case["kv_heads"]
    if op == "token":
        out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        for i, length in enumerate(_lengths(case)):
            at = torch.arange(length, device="cuda")
            rows = s["pages"][i].long()[at // case["page"]] * case["page"] + at % case["page"]
            for h in range(case["kv_heads"]):
                k, v = (s[name].flatten(0, 1)[rows, h].double() for name in ("k_cache", "v_cache"))
                mine = slice(h * group, (h + 1) * group)
                out[i, mine] = torch.softmax(s["scale"] * (s["q"][i, mine].double() @ k.t()), 1) @ v
        return out
    if work(case)["flops"] > 4e12:
        return None
    out = {name: torch.zeros(s[name].shape, dtype=torch.float64, device="cuda") for name in "qkv"}
    lse = torch.empty(case["heads"], s["q"].shape[0], dtype=torch.float64, device="cuda")
    q_at, k_at = s["on_host"]
    for i in range(len(q_at) - 1):
        lq, keys = q_at[i + 1] - q_at[i], slice(k_at[i], k_at[i + 1])
        step = max(1, (1 << 27) // max(1, k_at[i + 1] - k_at[i]))
        for head in range(case["heads"]):
            h = head // group
            k, v = s["k"][keys, h].double(), s["v"][keys, h].double()
            for lo in range(0, lq, step):
                hi = min(lq, lo + step)
                rows = slice(q_at[i] + lo, q_at[i] + hi)
                x, total = _weights_64(s, i, head, group, lo, hi)
                if op == "prompt":
                    out["q"][rows, head] = torch.exp(x - total[:, None]) @ v
                    lse[head, rows] = total
                    continue
                # the statistics and output that the forward pass gave are inputs of the gradients
                p = torch.exp(x - s["lse"][head, rows].double()[:, None])
                dout = s["dout"][rows, head].double()
                along = torch.linalg.vecdot(dout, s["out"][rows, head].double())
                ds = s["scale"] * p * (dout @ v.t() - along[:, None])
                out["q"][rows, head] = ds @ k
                out["k"][keys, h] += ds.t() @ s["q"][rows, head].double()
                out["v"][keys, h] += p.t() @ dout
    if op == "prompt":
        return {"out": out["q"], "lse": lse}
    return {"dq": out["q"], "dk": out["k"], "dv": out["v"]}
