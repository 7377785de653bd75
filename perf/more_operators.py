"""The operators that make rollouts and their cases: products with 4-bit weights, tokens drawn from logits, and verification of
drafted tokens, each in its plain form and as the framework's call.

  matvec  w_ij = scale_ig (code_ij - zero_ig) with g = j // group (no zeros: 8);  y_ri = sum_j w_ij x_rj.
  draw    p = softmax(z / temperature) of a row; with u in [0, 1) the token is the smallest j with p_0 + .. + p_j > u; its log p.
  verify  a request has K drafted tokens x_t, the drafter's distributions q_t (none: all of it on x_t) and the target's p_0 .. p_K.
          x_t is accepted if q_t(x_t) > 0 and u_t q_t(x_t) < p_t(x_t).  At the first that is not, a token is drawn from
          max(p_t - q_t, 0), after all of them one from p_K, by another number v.  The target's log-probabilities of what is emitted."""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one token through a small projection: the length of one call
        dict(name="matvec_small", op="matvec", x="bf16", y="bf16", rows=1, n=4096, k=2048, group=64, scale="bf16", zero=False),
        # one token through a large head, the ordinary step of a drafter
        dict(name="matvec_head", op="matvec", x="bf16", y="bf16", rows=1, n=131072, k=4096, group=128, scale="bf16", zero=False),
        # a few requests, sizes that no power of two divides, a last group that ends early
        dict(name="matvec_ragged", op="matvec", x="f16", y="f16", rows=5, n=50021, k=2600, group=128, scale="f16", zero=True),
        # activations in 32 bits and small groups
        dict(name="matvec_f32", op="matvec", x="f32", y="f32", rows=3, n=32768, k=2048, group=32, scale="f32", zero=True),
        # the drafts of a dozen requests at once, logits in 32 bits
        dict(name="matvec_batch", op="matvec", x="bf16", y="f32", rows=48, n=65536, k=4096, group=128, scale="f16", zero=True),
        # the next token of a few running requests
        dict(name="draw_decode", op="draw", dtype="bf16", rows=8, vocab=32768, temperature=0.8),
        # rollouts from given prompts, a vocabulary that no power of two divides
        dict(name="draw_ragged", op="draw", dtype="f16", rows=1001, vocab=50021, temperature=1.0),
        # a large batch of positions
        dict(name="draw_large", op="draw", dtype="bf16", rows=8192, vocab=131072, temperature=1.0),
        # two requests, tokens drafted without a distribution
        dict(name="verify_small", op="verify", dtype="bf16", requests=2, drafts=3, vocab=32768, drafter=False, logp=False, short=0.0,
             temperature=1.0, draft_temperature=1.0),
        # an ordinary step: the drafter's log-probabilities are at hand
        dict(name="verify_step", op="verify", dtype="bf16", requests=32, drafts=4, vocab=131072, drafter=True, logp=True, short=0.0,
             temperature=0.8, draft_temperature=0.8),
        # requests with fewer drafts than others, in 32 bits, from the two sides' logits alone
        dict(name="verify_ragged", op="verify", dtype="f32", requests=37, drafts=6, vocab=50021, drafter=True, logp=False, short=0.4,
             temperature=1.0, draft_temperature=1.2),
        # a large batch
        dict(name="verify_large", op="verify", dtype="f16", requests=256, drafts=5, vocab=131072, drafter=True, logp=True, short=0.0,
             temperature=1.0, draft_temperature=1.0),
    ]


def draw(rng):
    def spread(low, high):
        return int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))

    op = rng.choice(("matvec", "draw", "verify"))
    if op == "matvec":
        rows = spread(1, 64)
        k = spread(64, 8192)
        n = spread(64, min(131072, (1 << 29 if rows <= 16 else 1 << 28) // k))
        x = rng.choice(("f32", "bf16", "f16"))
        return dict(op=op, x=x, y=rng.choice((x, "f32")), rows=rows, n=n, k=k, group=rng.choice((32, 64, 128)),
                    scale=rng.choice(("f32", "bf16", "f16")), zero=rng.random() < 0.5)
    dtype = rng.choice(("f32", "bf16", "f16"))
    vocab = spread(1000, 140000)
    if op == "draw":
        rows = spread(1, max(1, min(8192, int(2.1e9 / (SIZE[dtype] * vocab)))))
        return dict(op=op, dtype=dtype, rows=rows, vocab=vocab, temperature=rng.choice((0.7, 1.0)))
    drafts = spread(1, 8)
    requests = spread(1, max(1, min(256, int(4.0e8 / (SIZE[dtype] * vocab * (drafts + 1))))))
    drafter = rng.random() < 0.75
    return dict(op=op, dtype=dtype, requests=requests, drafts=drafts, vocab=vocab, drafter=drafter, logp=drafter and rng.random() < 0.5,
                short=rng.choice((0.0, 0.4)), temperature=rng.choice((0.7, 1.0)), draft_temperature=rng.choice((0.8, 1.0)))


# The share of drafted tokens that is accepted, one after another, with the inputs below: of a drafter near the target, and of likely tokens.
ACCEPTED = {True: 0.85, False: 0.4}


def work(case):
    if case["op"] == "matvec":
        n, k, rows = case["n"], case["k"], case["rows"]
        groups = -(-k // case["group"])
        return {"bytes": n * -(-k // 2) + n * groups * SIZE[case["scale"]] * (1 + case["zero"]) + rows * (k * SIZE[case["x"]] + n * SIZE[case["y"]]),
                "flops": 2 * rows * n * k}
    vocab, b = case["vocab"], SIZE[case["dtype"]]
    if case["op"] == "draw":
        return {"bytes": case["rows"] * (vocab * b + 4 + 8 + 4), "flops": 4 * case["rows"] * vocab}
    n, drafts = case["requests"], case["drafts"] * (1 - case["short"] / 2)
    accepted = ACCEPTED[case["drafter"]]
    target = sum(accepted ** t for t in range(round(drafts) + 1))        # rows of the target up to the first refusal
    refused = 1 - accepted ** drafts
    drafter = 0 if not case["drafter"] else refused if case["logp"] else min(drafts, target)
    small = case["drafts"] * (8 + 4 + 4 * case["logp"]) + 4 + (case["drafts"] + 1) * (8 + 4) + 8
    return {"bytes": int(n * ((target + drafter) * vocab * b + small)), "flops": int(n * (target + 2 * drafter) * 4 * vocab)}


# ---- inputs ---------------------------------------------------------------------------------------------------------------


def _clear_number(cdf, gen, margin):
    """A number u in [0, 1) for each row of running sums (in 64 bits) whose u * total is `margin` away from every one of them: which token a
    number on the border stands for is a matter of rounding, so none is there."""
    rows = cdf.shape[0]
    u = torch.rand(rows, 64, device=DEV, generator=gen)
    at = u.double() * cdf[:, -1:]
    j = torch.searchsorted(cdf, at, right=True).clamp(max=cdf.shape[1] - 1)
    above = cdf.gather(1, j) - at
    below = at - torch.where(j > 0, cdf.gather(1, (j - 1).clamp(min=0)), -1.0)
    room = torch.minimum(above, below)
    pick = torch.where((room >= margin).any(1), (room >= margin).int().argmax(1), room.argmax(1))
    return u.gather(1, pick[:, None])[:, 0].contiguous()


MARGIN = 4e-7


def _logits(shape, dtype, gen):
    """Logits as a model gives them: most of the mass on a few dozen entries, the rest spread wide."""
    vocab = shape[-1]
    z = torch.empty(*shape, dtype=dtype, device=DEV)
    flat = z.view(-1, vocab)
    for a in range(0, len(flat), 1024):
        part = torch.randn(min(1024, len(flat) - a), vocab, device=DEV, generator=gen).mul_(2.2)
        first = torch.randint(0, vocab, (len(part), 1), device=DEV, generator=gen)
        stride = torch.randint(1, vocab // 24, (len(part), 1), device=DEV, generator=gen)     # (so that no index comes twice)
        top = (first + stride * torch.arange(24, device=DEV)) % vocab
        part.scatter_(1, top, math.log(vocab) + 1.0 + 1.5 * torch.randn(len(part), 24, device=DEV, generator=gen))
        flat[a:a + 1024] = part
    return z


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    st = dict(case=case)

    def randn(*shape):
        return torch.randn(*shape, device=DEV, generator=gen)

    def rand(*shape):
        return torch.rand(*shape, device=DEV, generator=gen)

    if case["op"] == "matvec":
        n, k, groups = case["n"], case["k"], -(-case["k"] // case["group"])
        wide = -(-k // 2)
        codes = torch.empty(n, wide, dtype=torch.uint8, device=DEV)      # two codes a byte, the even column's in the low four bits
        for a in range(0, n, 8192):
            rows = min(8192, n - a)
            low, high = (randn(rows, wide).mul_(2.7).add_(7.5).round_().clamp_(0, 15).to(torch.uint8) for _ in range(2))
            if k % 2:
                high[:, -1] = 0
            codes[a:a + rows] = low | high << 4
        st["codes"] = codes
        st["scale"] = (0.006 * (0.5 + rand(n, groups))).to(TYPES[case["scale"]])
        st["zero"] = torch.randint(6, 10, (n, groups), device=DEV, generator=gen).to(TYPES[case["scale"]]) if case["zero"] else None
        st["x"] = randn(case["rows"], k).to(TYPES[case["x"]])
        if own:
            import paper_2203_16340_amd as L
            st["w"] = L.pack4(codes, st["scale"], st["zero"], cols=k, group=case["group"])
        return st
    dtype, vocab = TYPES[case["dtype"]], case["vocab"]
    if case["op"] == "draw":
        z = st["z"] = _logits((case["rows"], vocab), dtype, gen)
        st["u"] = torch.cat([_clear_number(torch.cumsum(torch.softmax(z[a:a + 512].double() / case["temperature"], 1), 1), gen, MARGIN)
                             for a in range(0, case["rows"], 512)])
        return st
    n, K = case["requests"], case["drafts"]
    z = st["z"] = _logits((n, K + 1, vocab), dtype, gen)
    length = None
    if case["short"]:
        length = torch.where(rand(n) < case["short"], torch.randint(0, K + 1, (n,), device=DEV, generator=gen), K)
    st["length"] = length
    steps = torch.arange(K, device=DEV)
    s, sq = 1.0 / case["temperature"], 1.0 / case["draft_temperature"]
    drafted, draft_logp = torch.empty(n, K, dtype=torch.int64, device=DEV), torch.empty(n, K, device=DEV)
    u, v = torch.empty(n, K, device=DEV), torch.empty(n, device=DEV)
    zq = torch.empty(n, K, vocab, dtype=dtype, device=DEV) if case["drafter"] else None
    chunk = max(1, int(4e8) // (8 * vocab * (K + 1)))
    for a in range(0, n, chunk):
        at = slice(a, min(a + chunk, n))
        p = torch.softmax(z[at].double() * s, 2)
        m = len(p)
        if case["drafter"]:                                              # a drafter near the target
            zq[at] = (z[at, :K].float() * (case["draft_temperature"] * s) + 0.45 * randn(m, K, vocab)).to(dtype)
            q = torch.softmax(zq[at].double() * sq, 2)
            x = torch.searchsorted(torch.cumsum(q, 2), rand(m, K, 1).double() * q.sum(2, keepdim=True), right=True).clamp(max=vocab - 1)
            qx = q.gather(2, x)[..., 0]
        else:                                                            # or one that proposes likely tokens, and now and then another
            x = torch.where(rand(m, K, 1) < 0.9, p[:, :K].argmax(2, keepdim=True), torch.randint(0, vocab, (m, K, 1), device=DEV, generator=gen))
            q = torch.zeros_like(p[:, :K]).scatter_(2, x, 1.0)
            qx = torch.ones(m, K, dtype=torch.float64, device=DEV)
        ratio = p[:, :K].gather(2, x)[..., 0] / qx
        draw_u = rand(m, K)
        if not case["drafter"]:                                          # (proposals that are likelier than the logits make them look)
            draw_u = draw_u * (0.4 + 0.6 * rand(m, K))
        draw_u = torch.where((draw_u - ratio).abs() < 1e-4, (draw_u - 3e-4).abs(), draw_u)     # none on the border
        u[at], drafted[at], draft_logp[at] = draw_u, x[..., 0], torch.log(qx).float()
        here = torch.full((m,), K, device=DEV) if length is None else length[at]
        good = (draw_u.double() * qx < p[:, :K].gather(2, x)[..., 0]) & (steps < here[:, None])
        count = torch.cumprod(good.int(), 1).sum(1)
        each = torch.arange(m, device=DEV)
        rest = p[each, count]
        refused = count < here
        rest = torch.where(refused[:, None], (rest - q[each, count.clamp(max=K - 1)]).clamp(min=0), rest)
        v[at] = _clear_number(torch.cumsum(rest, 1), gen, MARGIN)
    st.update(zq=zq, drafted=drafted, logp=draft_logp if case["logp"] else None, u=u, v=v)
    return st


# ---- one pass -------------------------------------------------------------------------------------------------------------


def run(st):
    case = st["case"]
    return _framework(st, case) if own else PLAIN[case["op"]](st, case)


def _framework(st, case):
    import paper_2203_16340_amd as L
    if case["op"] == "matvec":
        return L.matvec4(st["x"], st["w"], dtype=TYPES[case["y"]])
    if case["op"] == "draw":
        r = L.draw_tokens(st["z"], st["u"], temperature=case["temperature"])
        return {"tokens": r.tokens, "logp": r.logp}
    r = L.verify_draft(st["z"], st["drafted"], st["u"], st["v"], draft_logits=st["zq"], draft_logp=st["logp"], lengths=st["length"],
                       temperature=case["temperature"], draft_temperature=case["draft_temperature"])
    return {"tokens": r.tokens, "count": r.count, "logp": r.logp}


def _plain_matvec(st, case):
    k, group = case["k"], case["group"]
    codes, scale, zero = st["codes"], st["scale"].float(), st["zero"]
    code = torch.stack([codes & 15, codes >> 4], 2).flatten(1)[:, :k].float()
    of = torch.arange(k, device=DEV) // group
    w = (code - (8.0 if zero is None else zero.float()[:, of])) * scale[:, of]
    return (st["x"].float() @ w.t()).to(TYPES[case["y"]])


def _plain_draw(st, case):
    """(probabilities and their sums in 64 bits: a number next to a token's border has to fall on its side of it)"""
    z, u = st["z"], st["u"]
    tokens, logp = [], []
    for a in range(0, len(z), 1024):
        y = z[a:a + 1024].double() / case["temperature"]
        y = y - y.amax(1, keepdim=True)
        e = torch.exp(y)
        running = torch.cumsum(e, 1)
        total = running[:, -1:]
        at = (running <= u[a:a + 1024, None].double() * total).sum(1)
        tokens.append(at)
        logp.append((y.gather(1, at[:, None]) - torch.log(total))[:, 0].float())
    return {"tokens": torch.cat(tokens), "logp": torch.cat(logp)}


def _plain_softmax(z, s):
    y = z.double() * s
    e = torch.exp(y - y.amax(2, keepdim=True))
    return e / e.sum(2, keepdim=True)


def _plain_verify(st, case):
    n, K, vocab = case["requests"], case["drafts"], case["vocab"]
    z, zq, sq = st["z"], st["zq"], 1.0 / case["draft_temperature"]
    steps = torch.arange(K + 1, device=DEV)
    out = []
    chunk = max(1, int(1.5e9) // (8 * vocab * (K + 1)))
    for a in range(0, n, chunk):
        at = slice(a, a + chunk)
        p = _plain_softmax(z[at], 1.0 / case["temperature"])
        m = len(p)
        x = st["drafted"][at][..., None]
        if zq is None:
            q = torch.zeros_like(p[:, :K]).scatter_(2, x, 1.0)
        elif st["logp"] is None:
            q = _plain_softmax(zq[at], sq)
        else:
            y = zq[at].double() * sq
            q = torch.exp(y - y.gather(2, x) + st["logp"][at].double()[..., None])
        length = torch.full((m,), K, device=DEV) if st["length"] is None else st["length"][at]
        px, qx = p[:, :K].gather(2, x)[..., 0], q.gather(2, x)[..., 0]
        good = (qx > 0) & (st["u"][at].double() * qx < px) & (steps[:K] < length[:, None])
        count = torch.cumprod(good.int(), 1).sum(1)
        each = torch.arange(m, device=DEV)
        last = p[each, count]
        rest = torch.where((count < length)[:, None], (last - q[each, count.clamp(max=K - 1)]).clamp(min=0), last)
        running = torch.cumsum(rest, 1)
        final = (running <= st["v"][at].double()[:, None] * running[:, -1:]).sum(1)
        tokens = torch.cat([st["drafted"][at], final[:, None]], 1)
        tokens = torch.where(steps < count[:, None], tokens, torch.where(steps == count[:, None], final[:, None], -1))
        logp = torch.log(p.gather(2, tokens.clamp(min=0)[..., None])[..., 0])
        out.append((tokens, count + 1, torch.where(tokens < 0, 0.0, logp).float()))
    tokens, count, logp = (torch.cat(t) for t in zip(*out))
    return {"tokens": tokens, "count": count, "logp": logp}


PLAIN = {"matvec": _plain_matvec, "draw": _plain_draw, "verify": _plain_verify}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------------


def exact(case, seed):
    st = prepare(case, seed)
    return {"matvec": _exact_matvec, "draw": _exact_draw, "verify": _exact_verify}[case["op"]](st, case)


def _exact_matvec(st, case):
    x, k, group = st["x"].double(), case["k"], case["group"]
    parts = []
    for a in range(0, case["n"], 8192):
        byte = st["codes"][a:a + 8192]
        w = torch.empty(len(byte), 2 * byte.shape[1], dtype=torch.float64, device=DEV)
        w[:, 0::2], w[:, 1::2] = byte % 16, byte // 16
        w = w[:, :k]
        for g in range(-(-k // group)):
            of = slice(g * group, min((g + 1) * group, k))
            w[:, of] -= 8.0 if st["zero"] is None else st["zero"][a:a + 8192, g:g + 1].double()
            w[:, of] *= st["scale"][a:a + 8192, g:g + 1].double()
        parts.append(torch.mm(x, w.t().contiguous()))
    return torch.cat(parts, 1)


def _exact_draw(st, case):
    tokens, logp = [], []
    for a in range(0, case["rows"], 256):
        lp = torch.log_softmax(st["z"][a:a + 256].double() / case["temperature"], 1)
        cdf = torch.cumsum(lp.exp(), 1)
        j = torch.searchsorted(cdf, st["u"][a:a + 256, None].double() * cdf[:, -1:], right=True)
        tokens.append(j[:, 0])
        logp.append(lp.gather(1, j)[:, 0])
    return {"tokens": torch.cat(tokens), "logp": torch.cat(logp)}


def _exact_verify(st, case):
    n, K = case["requests"], case["drafts"]
    tokens = torch.full((n, K + 1), -1, dtype=torch.int64, device=DEV)
    logp = torch.zeros(n, K + 1, dtype=torch.float64, device=DEV)
    count = torch.zeros(n, dtype=torch.int64, device=DEV)
    length = [K] * n if st["length"] is None else st["length"].tolist()
    drafted, u, v = st["drafted"].tolist(), st["u"].tolist(), st["v"].tolist()
    sq = 1.0 / case["draft_temperature"]
    for i in range(n):
        lp = torch.log_softmax(st["z"][i].double() / case["temperature"], 1)
        t, rest = 0, None
        while True:
            if t == length[i]:
                rest = lp[t].exp()
                break
            x = drafted[i][t]
            if st["zq"] is None:
                q = torch.zeros_like(lp[t])
                q[x] = 1
            elif st["logp"] is None:
                q = torch.log_softmax(st["zq"][i, t].double() * sq, 0).exp()
            else:
                q = ((st["zq"][i, t].double() - st["zq"][i, t, x].double()) * sq + st["logp"][i, t].double()).exp()
            qx, px = float(q[x]), float(lp[t, x].exp())
            if not (qx > 0 and u[i][t] * qx < px):
                rest = torch.relu(lp[t].exp() - q)
                break
            tokens[i, t], logp[i, t] = x, lp[t, x]
            t += 1
        cdf = torch.cumsum(rest, 0)
        j = int(torch.searchsorted(cdf, (cdf[-1] * v[i]).reshape(1), right=True))
        tokens[i, t], logp[i, t], count[i] = j, lp[t, j], t + 1
    return {"tokens": tokens, "count": count, "logp": logp}
