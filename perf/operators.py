"""What is timed of the operators for batches of text turns and for the key/value cache that their answers are read from.

Four paths, each through the public entry points of ``paper_2604_08077_amd.binding`` where ``own`` is true, and in
elementary torch operations where it is not:

  prompt   causal attention over packed prompts of different lengths; with more keys than queries, over a follow-up turn
  train    the same with the log-sum-exp, then its gradients: one attention layer of a training step
  cache    the keys and values of new tokens written into a paged cache, whole histories read back from it, or both
  decode   attention of one new token of each sequence over its pages

Heads and head sizes are those of the repository's benchmark and test workloads, lengths go from one token to the tens of
thousands of a long video's prompt.
"""
import math

import torch

own = False

# A case: "path"; Hq, Hkv, D; "q": the sequences' lengths in query tokens (prompt, train) or in new tokens (cache), with
# commas; "k": their lengths in keys, or in tokens of the cache after the new ones ("": as many as queries); for the
# cache and decode also "page", tokens of a page, and "format", "bf16" or "e4m3"; for the cache "do": "write" (bf16 only: what
# 8 bits hold is compared by the values read back), "read" or "both".


def _case(name, path, heads, q, k="", **more):
    c = {"name": name, "path": path, "Hq": heads[0], "Hkv": heads[1], "D": heads[2], "q": q, "k": k}
    c.update(more)
    return c


def listed():
    return [
        # a handful of short questions in one batch through a small model: the latency of a call
        _case("prompt short", "prompt", (4, 4, 64), "37,1,120,5,64,73"),
        # a serving batch of sixteen prompts, none a whole number of tiles
        _case("prompt 8k in 16", "prompt", (28, 4, 128),
              "1201,33,760,512,95,1,250,1033,407,61,888,129,333,1504,17,960"),
        # follow-up questions about long videos: few queries on what the cache gave back
        _case("prompt follow-up", "prompt", (32, 8, 128), "301,77", "20301,9077"),
        # one long prompt in the backbone's heads
        _case("prompt 32k", "prompt", (28, 4, 128), "32001"),
        # training on short dialogues, packed; and on long ones
        _case("train 2k in 3", "train", (8, 2, 64), "700,1,1323"),
        _case("train 16k in 5", "train", (28, 4, 128), "6000,4096,3500,1999,800"),
        # a turn of a small model written into its cache
        _case("cache write 1k", "cache", (4, 4, 64), "300,1,700", "812,1,700", page=16, format="bf16", do="write"),
        # a prefill of several prompts written in 8 bits, and the histories read back for the attention that follows
        _case("cache both 24k e4m3", "cache", (28, 4, 128), "8000,3001,5000,77", "8000,9001,6200,1077", page=64,
              format="e4m3", do="both"),
        # long histories read back for a follow-up turn
        _case("cache read 64k e4m3", "cache", (32, 8, 128), "0,0,0", "40001,20000,5535", page=64, format="e4m3", do="read"),
        # answers: one sequence in a short chat; a ragged batch on an 8-bit cache; long videos
        _case("decode one 2k", "decode", (28, 4, 128), "1", "2049", page=16, format="bf16"),
        _case("decode 32 ragged e4m3", "decode", (32, 8, 128), ",".join(["1"] * 32),
              ",".join(str(1 + (i * i * 37 + 911 * i) % 12000) for i in range(32)), page=64, format="e4m3"),
        _case("decode 8 of 60k", "decode", (28, 4, 128), ",".join(["1"] * 8),
              "65536,60001,33333,64000,48123,65001,59999,50017", page=64, format="bf16"),
    ]


def _near(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _ragged(rng, total, count, most):
    """count lengths of at least 1 that sum to about total, few of them long."""
    w = [math.exp(rng.uniform(0, 3)) for _ in range(count)]
    return [max(1, min(most, int(total * x / sum(w)))) for x in w]


def draw(rng):
    path = rng.choice(("prompt", "prompt", "train", "cache", "cache", "decode", "decode"))
    heads = rng.choice(((4, 4, 64), (8, 2, 64), (6, 2, 128), (28, 4, 128), (28, 4, 128), (32, 8, 128), (12, 3, 128), (16, 16, 64)))
    join = lambda v: ",".join(str(x) for x in v)  # noqa: E731
    if path in ("prompt", "train"):
        total = _near(rng, 64, 24000 if path == "prompt" else 12000)
        count = rng.randint(1, min(24, 1 + total // 40))
        q = _ragged(rng, total, count, 24000)
        k = ""
        if path == "prompt" and rng.random() < 0.4:  # turns on a history
            q = [min(x, _near(rng, 1, 800)) for x in q]
            k = join(x + rng.choice((0, _near(rng, 16, 24000 // count))) for x in q)
        return {"path": path, "Hq": heads[0], "Hkv": heads[1], "D": heads[2], "q": join(q), "k": k}
    page, fmt = rng.choice((16, 32, 64, 128, 256)), rng.choice(("bf16", "e4m3"))
    count = rng.randint(1, 32)
    k = _ragged(rng, _near(rng, 200, 60000 if path == "cache" else 200000), count, 65536)
    if path == "cache":
        do = rng.choice(("write" if fmt == "bf16" else "both", "read", "both"))
        q = [0] * count if do == "read" else [min(x, _near(rng, 1, 8000)) for x in k]
        return {"path": path, "Hq": heads[0], "Hkv": heads[1], "D": heads[2], "q": join(q), "k": join(k), "page": page,
                "format": fmt, "do": do}
    return {"path": path, "Hq": heads[0], "Hkv": heads[1], "D": heads[2], "q": join([1] * count), "k": join(k),
            "page": page, "format": fmt}


def _lengths(case):
    q = [int(x) for x in case["q"].split(",")]
    return q, [int(x) for x in case["k"].split(",")] if case["k"] else list(q)


def _pairs(case):
    """Attended (query token, key) pairs of one head: token i of n on m keys attends i + m - n + 1 of them."""
    q, k = _lengths(case)
    return sum(n * (m - n) + n * (n + 1) // 2 for n, m in zip(q, k))


def work(case):
    q, k = _lengths(case)
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    tq, tk = sum(q), sum(k)
    if case["path"] == "prompt":
        return {"bytes": 4 * tq * Hq * D + 4 * tk * Hkv * D, "flops": 4 * D * Hq * _pairs(case)}
    if case["path"] == "train":  # forward and backward: Q, K, V, dO in, O, lse, dQ, dK, dV out; 2 + 5 products
        return {"bytes": 8 * tq * Hq * D + 8 * tk * Hkv * D + 4 * tq * Hq, "flops": 14 * D * Hq * _pairs(case)}
    row = 2 * Hkv * (D + 4 if case["format"] == "e4m3" else 2 * D)  # K and V of a token in the cache
    if case["path"] == "decode":
        return {"bytes": tk * row + 4 * len(q) * Hq * D, "flops": 4 * D * Hq * tk}
    moved = {"write": tq * (4 * Hkv * D + row), "read": tk * (4 * Hkv * D + row)}
    return {"bytes": moved["write"] + moved["read"] if case["do"] == "both" else moved[case["do"]], "flops": 0}


def _starts(lengths):
    s = [0]
    for n in lengths:
        s.append(s[-1] + n)
    return torch.tensor(s, dtype=torch.int32, device="cuda")


def _pool(g, pages, page, Hkv, D, fmt):
    """A cache in use: [pages][KV heads][tokens of a page][D], in 8 bits with a scale for each token and head."""
    pool = []
    for _ in range(2):
        x = torch.randn((pages, Hkv, page, D), generator=g, device="cuda", dtype=torch.float32)
        if fmt == "bf16":
            pool.append((x.to(torch.bfloat16), None))
        else:
            scale = x.abs().amax(-1) / 448
            pool.append(((x / scale[..., None]).to(torch.float8_e4m3fn), scale.contiguous()))
        del x
    return pool


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    q, k = _lengths(case)
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)

    s = dict(case, q_len=q, k_len=k)
    if case["path"] in ("prompt", "train"):
        s["q_start"], s["k_start"] = _starts(q), _starts(k)
        s["Q"] = randn(sum(q), Hq, D).to(torch.bfloat16)
        # keys that share a direction, as those of one text do
        s["K"] = (randn(sum(k), Hkv, D) + randn(1, Hkv, D)).to(torch.bfloat16)
        s["V"] = randn(sum(k), Hkv, D).to(torch.bfloat16)
        if case["path"] == "train":
            s["dO"] = randn(sum(q), Hq, D).to(torch.bfloat16)
        return s
    page = case["page"]
    need = [(m + page - 1) // page for m in k]
    pages = sum(need) + 3
    table_pages = max(need) + 1
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(k), table_pages), -1, dtype=torch.int32)  # past a sequence's pages: none
    order_h, at = order.cpu(), 0
    for b, n in enumerate(need):
        table[b, :n] = order_h[at:at + n]
        at += n
    s.update(pages=pages, table_pages=table_pages, table=table.cuda(),
             lengths=torch.tensor(k, dtype=torch.int32, device="cuda"))
    (s["Kc"], s["ks"]), (s["Vc"], s["vs"]) = _pool(g, pages, page, Hkv, D, case["format"])
    if case["path"] == "decode":
        s["Q"] = randn(len(q), Hq, D).to(torch.bfloat16)
    else:
        s["q_start"], s["k_start"] = _starts(q), _starts(k)
        s["K"], s["V"] = randn(sum(q), Hkv, D).to(torch.bfloat16), randn(sum(q), Hkv, D).to(torch.bfloat16)
    return s


def _written(s):
    """What a write leaves: the cache itself, or the scales of one in 8 bits, whose codes come out as the values read back."""
    return {"K": s["Kc"], "V": s["Vc"]} if s["format"] == "bf16" else {"ks": s["ks"], "vs": s["vs"]}


# ---- the operators as a user calls them


def _run_own(s):
    from paper_2604_08077_amd import binding as B

    if s["path"] in ("prompt", "train"):
        sh = B.PromptShape(len(s["q_len"]), s["Q"].shape[0], s["K"].shape[0], s["Hq"], s["Hkv"], s["D"])
        if s["path"] == "prompt":
            return B.prompt_attn(sh, s["Q"], s["K"], s["V"], s["q_start"], s["k_start"])
        O, lse = B.prompt_attn(sh, s["Q"], s["K"], s["V"], s["q_start"], s["k_start"], return_lse=True)
        dQ, dK, dV = B.prompt_attn_bwd(sh, s["Q"], s["K"], s["V"], O, lse, s["dO"], s["q_start"], s["k_start"])
        return {"O": O, "lse": lse, "dQ": dQ, "dK": dK, "dV": dV}
    sh = B.CacheShape(len(s["q_len"]), s["pages"], s["page"], s["table_pages"], s["Hq"], s["Hkv"], s["D"], s["format"])
    cache = B.Cache(s["Kc"], s["Vc"], s["ks"], s["vs"])
    if s["path"] == "decode":
        return B.decode_attn(sh, s["Q"], cache, s["table"], s["lengths"])
    out = {}
    if s["do"] != "read":
        B.cache_write(sh, s["K"], s["V"], s["q_start"], cache, s["table"], s["lengths"])
        out.update(_written(s))
    if s["do"] != "write":
        out["K"], out["V"] = B.cache_read(sh, cache, s["table"], s["k_start"], sum(s["k_len"]))
    return out


# ---- their plain form


CHUNK = 1 << 28  # scores worked at a time


def _plain_scores(q, k, first, Hkv):
    """Rows (token, head of a group) of every KV head: their scaled scores against k, -inf behind a row's own position.
    q [n, Hq, D] fp32, k [Hkv, m, D] fp32; first: keys that the first token attends besides itself."""
    n, Hq, D = q.shape
    m = k.shape[1]
    rows = q.view(n, Hkv, Hq // Hkv, D).permute(1, 0, 2, 3).reshape(Hkv, -1, D)
    sc = torch.matmul(rows, k.transpose(1, 2).contiguous()) / math.sqrt(D)
    reach = first + torch.arange(n, device=q.device).repeat_interleave(Hq // Hkv)
    return rows, sc.masked_fill_(torch.arange(m, device=q.device) > reach[:, None], -math.inf)


def _plain_prompt(s, grads):
    Hq, Hkv, D = s["Hq"], s["Hkv"], s["D"]
    G = Hq // Hkv
    O = torch.empty_like(s["Q"])
    lse = torch.empty(s["Q"].shape[:2], dtype=torch.float32, device="cuda")
    out = {"O": O, "lse": lse}
    if grads:
        out.update(dQ=torch.empty_like(s["Q"]), dK=torch.empty_like(s["K"]), dV=torch.empty_like(s["V"]))
    q0 = k0 = 0
    tokens = lambda rows, n: rows.view(Hkv, n, G, -1).permute(1, 0, 2, 3).reshape(n, Hq, -1)  # noqa: E731
    for n, m in zip(s["q_len"], s["k_len"]):
        k = s["K"][k0:k0 + m].float().transpose(0, 1).contiguous()
        v = s["V"][k0:k0 + m].float().transpose(0, 1).contiguous()
        if grads:
            dk, dv = torch.zeros_like(k), torch.zeros_like(v)
        step = max(1, CHUNK // (Hq * m))
        for i in range(0, n, step):
            j = min(n, i + step)
            last = m - n + j  # keys that some row of the chunk attends
            kk, vv = k[:, :last], v[:, :last]
            rows, p = _plain_scores(s["Q"][q0 + i:q0 + j].float(), kk, m - n + i, Hkv)
            top = p.amax(-1, keepdim=True)
            p = p.sub_(top).exp_()
            total = p.sum(-1, keepdim=True)
            p = p.div_(total)
            O[q0 + i:q0 + j] = tokens(torch.matmul(p, vv), j - i)
            lse[q0 + i:q0 + j] = tokens(top + total.log(), j - i)[..., 0]
            if grads:
                go = s["dO"][q0 + i:q0 + j].float().view(j - i, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, -1, D)
                dv[:, :last] += torch.matmul(p.transpose(1, 2).contiguous(), go)
                dp = torch.matmul(go, vv.transpose(1, 2).contiguous())
                dp = dp.sub_((dp * p).sum(-1, keepdim=True)).mul_(p)
                out["dQ"][q0 + i:q0 + j] = tokens(torch.matmul(dp, kk) / math.sqrt(D), j - i)
                dk[:, :last] += torch.matmul(dp.transpose(1, 2).contiguous(), rows) / math.sqrt(D)
        if grads:
            out["dK"][k0:k0 + m] = dk.transpose(0, 1)
            out["dV"][k0:k0 + m] = dv.transpose(0, 1)
        q0, k0 = q0 + n, k0 + m
    return out if grads else O


def _plain_values(codes, scale, page, offset):
    """What the cache holds at (page, offset), both [...]: fp32 [..., Hkv, D]."""
    x = codes[page, :, offset].float()
    return x if scale is None else x * scale[page, :, offset][..., None]


def _plain_place(s, seq, pos):
    return s["table"][seq, pos // s["page"]].long(), pos % s["page"]


def _plain_cache(s):
    out = {}
    if s["do"] != "read":
        t = torch.arange(s["K"].shape[0], device="cuda")
        seq = torch.searchsorted(s["q_start"], t, right=True) - 1
        page, offset = _plain_place(s, seq, s["lengths"].long()[seq] - s["q_start"].long()[seq + 1] + t)
        for new, codes, scale in ((s["K"], s["Kc"], s["ks"]), (s["V"], s["Vc"], s["vs"])):
            if scale is None:
                codes[page, :, offset] = new
            else:
                x = new.float()
                sc = x.abs().amax(-1) / 448
                codes.view(torch.uint8)[page, :, offset] = (x / sc[..., None]).to(codes.dtype).view(torch.uint8)
                scale[page, :, offset] = sc
        out.update(_written(s))
    if s["do"] != "write":
        t = torch.arange(sum(s["k_len"]), device="cuda")
        seq = torch.searchsorted(s["k_start"], t, right=True) - 1
        page, offset = _plain_place(s, seq, t - s["k_start"].long()[seq])
        out["K"] = _plain_values(s["Kc"], s["ks"], page, offset).to(torch.bfloat16)
        out["V"] = _plain_values(s["Vc"], s["vs"], page, offset).to(torch.bfloat16)
    return out


def _plain_decode(s):
    B, Hq, D = s["Q"].shape
    Hkv, most = s["Hkv"], max(s["k_len"])
    O = torch.empty_like(s["Q"])
    step = max(1, (1 << 28) // (Hkv * most * D))
    pos = torch.arange(most, device="cuda")
    for b in range(0, B, step):
        q = s["Q"][b:b + step].float().view(-1, Hkv, Hq // Hkv, D)
        n = q.shape[0]
        seq = torch.arange(b, b + n, device="cuda")[:, None]
        page, offset = _plain_place(s, seq, pos[None])
        page = page.clamp_(min=0)  # (behind a sequence's pages: masked below)
        k = _plain_values(s["Kc"], s["ks"], page, offset).permute(0, 2, 3, 1).contiguous()  # [n, Hkv, D, most]
        sc = torch.matmul(q, k) / math.sqrt(D)
        del k
        sc = sc.masked_fill_(pos >= s["lengths"][b:b + n, None, None, None], -math.inf)
        p = sc.sub_(sc.amax(-1, keepdim=True)).exp_()
        p = p.div_(p.sum(-1, keepdim=True))
        v = _plain_values(s["Vc"], s["vs"], page, offset).transpose(1, 2).contiguous()
        O[b:b + n] = torch.matmul(p, v).view(n, Hq, D)
        del v
    return O


def run(state):
    if own:
        return _run_own(state)
    if state["path"] == "cache":
        return _plain_cache(state)
    if state["path"] == "decode":
        return _plain_decode(state)
    return _plain_prompt(state, state["path"] == "train")


# ---- the definitions in 64 bits


def _exact_e4m3(x):
    """The nearest e4m3 value, ties to even: 3 bits behind the leading one, exponents from -6, at most 448."""
    e = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -20))).clamp_min(-6.0)
    step = torch.exp2(e - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_attention(q, k, v, go, D):
    """One KV head, one sequence: q [n, G, D], k and v [m, D], 64 bits; the last query sees every key."""
    n, G, m = q.shape[0], q.shape[1], k.shape[0]
    o, lse = torch.empty_like(q), torch.empty(n, G, dtype=torch.float64, device=q.device)
    dq, dk, dv = torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)
    step = max(1, (1 << 27) // (G * m))
    for i in range(0, n, step):
        x = q[i:i + step]
        logits = torch.einsum("ngd,md->ngm", x, k) * D ** -0.5
        seen = torch.arange(m, device=q.device)[None] <= (m - n + torch.arange(i, i + len(x), device=q.device))[:, None]
        logits = torch.where(seen[:, None], logits, torch.full_like(logits, -math.inf))
        l = torch.logsumexp(logits, -1)
        w = torch.exp(logits - l[..., None])
        o[i:i + step], lse[i:i + step] = torch.einsum("ngm,md->ngd", w, v), l
        if go is not None:
            y = go[i:i + step]
            dv += torch.einsum("ngm,ngd->md", w, y)
            ds = w * (torch.einsum("ngd,md->ngm", y, v) - (y * o[i:i + step]).sum(-1, keepdim=True))
            dq[i:i + step] = torch.einsum("ngm,md->ngd", ds, k) * D ** -0.5
            dk += torch.einsum("ngm,ngd->md", ds, x) * D ** -0.5
    return o, lse, dq, dk, dv


def exact(case, seed):
    s = prepare(case, seed)
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    G = Hq // Hkv
    if case["path"] in ("prompt", "train"):
        train = case["path"] == "train"
        Q, K, V = (s[n].double() for n in ("Q", "K", "V"))
        dO = s["dO"].double() if train else None
        r = {n: torch.zeros_like(t) for n, t in (("O", Q), ("dQ", Q), ("dK", K), ("dV", V))}
        r["lse"] = torch.zeros(Q.shape[:2], dtype=torch.float64, device="cuda")
        a = b = 0
        for n, m in zip(s["q_len"], s["k_len"]):
            for h in range(Hkv):
                at = (slice(a, a + n), slice(h * G, (h + 1) * G))
                got = _exact_attention(Q[at], K[b:b + m, h], V[b:b + m, h], dO[at] if train else None, D)
                r["O"][at], r["lse"][at], r["dQ"][at], r["dK"][b:b + m, h], r["dV"][b:b + m, h] = got
            a, b = a + n, b + m
        return r if train else r["O"]
    page = case["page"]
    table = s["table"].cpu().tolist()
    held = {}
    for name, new in (("K", s.get("K")), ("V", s.get("V"))):
        codes, scale = s[name + "c"].double(), s["ks" if name == "K" else "vs"]
        scale = torch.ones(codes.shape[:3], dtype=torch.float64, device="cuda") if scale is None else scale.double()
        if case["path"] == "cache" and case["do"] != "read":
            a = 0
            for b, (n, m) in enumerate(zip(s["q_len"], s["k_len"])):
                for i in range(m - n, m):  # to the end of a page at a time
                    if i != m - n and i % page:
                        continue
                    j = min(m, (i // page + 1) * page)
                    x = new[a + i - (m - n):a + j - (m - n)].double().transpose(0, 1)  # [Hkv, tokens, D]
                    at = (table[b][i // page], slice(None), slice(i % page, i % page + j - i))
                    if case["format"] == "e4m3":
                        sc = x.abs().amax(-1) / 448
                        scale[at] = sc
                        x = _exact_e4m3(x / sc[..., None])
                    codes[at] = x
                a += n
        held[name] = (codes, scale)
    (kc, ks), (vc, vs) = held["K"], held["V"]

    def history(b, codes, scale):
        m = s["k_len"][b]
        at = torch.tensor(table[b][:(m + page - 1) // page], device="cuda")
        x = (codes[at] * scale[at][..., None]).transpose(0, 1)
        return x.reshape(Hkv, -1, D)[:, :m]

    if case["path"] == "decode":
        o = torch.empty(len(s["k_len"]), Hq, D, dtype=torch.float64, device="cuda")
        for b in range(len(s["k_len"])):
            k, v = history(b, kc, ks), history(b, vc, vs)
            x = s["Q"][b].double().view(Hkv, G, D)
            w = torch.exp(torch.log_softmax(torch.einsum("hgd,hmd->hgm", x, k) * D ** -0.5, -1))
            o[b] = torch.einsum("hgm,hmd->hgd", w, v).reshape(Hq, D)
        return o
    r = {}
    if case["do"] != "read":
        r.update(dict(K=kc, V=vc) if case["format"] == "bf16" else dict(ks=ks, vs=vs))
    if case["do"] != "write":
        for name, (codes, scale) in held.items():
            r[name] = torch.cat([history(b, codes, scale).transpose(0, 1) for b in range(len(s["k_len"]))])
    return r
