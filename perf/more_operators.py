"""Measured cases of the operators around the layers of a network: embedding, group norm with an activation, dropout.

Each is timed as its users drive it: ``fwd`` (a batch or a segment served), ``train`` (forward and all gradients), ``step`` (one
token for every sequence of a batch).  Activations lie as the framework's layers take them, [N, channels, positions]; where a
case says ``last``, channels lie next to each other in memory.  The plain forms are elementary torch operations in 32 bits,
long sums in 64.  ``exact`` is written from the definitions in 64 bits.
"""
import math

import torch

own = False


# ---- cases ------------------------------------------------------------------------------------------------------------
def _embed(name, use, dtype, N, D, L, V, scale=1.0, wide=True, ragged=False):
    return {"name": name, "op": "embed", "use": use, "dtype": dtype, "N": N, "D": D, "L": L, "V": V, "scale": scale, "wide": wide, "ragged": ragged}


def _norm(name, use, dtype, N, C, L, G, act="silu", last=False, ragged=False):
    return {"name": name, "op": "norm", "use": use, "dtype": dtype, "N": N, "C": C, "L": L, "G": G, "act": act, "last": last, "ragged": ragged}


def _dropout(name, dtype, N, C, L, p, residual=True, ragged=False):
    return {"name": name, "op": "dropout", "use": "train", "dtype": dtype, "N": N, "C": C, "L": L, "p": p, "residual": residual, "ragged": ragged}


def listed():
    return [
        # one token of 16 sequences: launch and host time are all of it
        _embed("embed_step_fp32_small", "step", "fp32", 16, 128, 1, 4096),
        # training on the genomics segments: five symbols, 15 channels, as bytes of text would be in 64-bit tokens
        _embed("embed_train_bf16_symbols", "train", "bf16", 16, 15, 60000, 5),
        # a padded batch in float of odd sizes, tokens of 32 bits
        _embed("embed_train_fp32_ragged", "train", "fp32", 12, 49, 4999, 257, 7.0, wide=False, ragged=True),
        # training at the sizes of the filter sweep (batch 8, 64 channels expanded twice, 20000 columns), six-letter words of four symbols
        _embed("embed_train_bf16_words", "train", "bf16", 8, 128, 20000, 4096, 128 ** 0.5),
        # a large vocabulary and many channels
        _embed("embed_train_bf16_wide", "train", "bf16", 8, 512, 8192, 32000),
        # a short window of two sequences: latency
        _norm("norm_fwd_fp32_small", "fwd", "fp32", 2, 32, 100, 8),
        # one whole segment of the genomics network's width, odd length, served
        _norm("norm_fwd_bf16_segment", "fwd", "bf16", 1, 15, 60001, 3, "relu"),
        # a padded batch in float, odd sizes
        _norm("norm_train_fp32_ragged", "train", "fp32", 6, 45, 4999, 5, "none", ragged=True),
        # training behind a layer of the filter sweep
        _norm("norm_train_bf16_sweep", "train", "bf16", 8, 64, 20000, 8, "relu"),
        # many channels, channels last
        _norm("norm_train_bf16_last", "train", "bf16", 8, 512, 8192, 32, last=True),
        # a padded batch of odd sizes in float
        _dropout("dropout_train_fp32_ragged", "fp32", 6, 45, 4999, 0.2, ragged=True),
        # the end of a residual block of the wide layer (batch 32, 256 channels, 8192 columns)
        _dropout("dropout_train_bf16_wide", "bf16", 32, 256, 8192, 0.1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw(rng):
    """Batches 1 ... 64, channels 1 ... 512, lengths 1 ... 60001, vocabularies 2 ... 32000, groups 1 ... channels."""
    op = rng.choice(("embed", "norm", "norm", "dropout"))
    N, L, dtype, ragged = _log_int(rng, 1, 64), _log_int(rng, 1, 60001), rng.choice(("fp32", "bf16")), rng.random() < 0.3
    most = 8 * 512 * 8192 // (1 if dtype == "bf16" else 2)
    if op == "norm":
        G = rng.choice((1, 2, 3, 4, 5, 8, 16, 32))
        C = G * _log_int(rng, 1, 512 // G)
        return _norm("", rng.choice(("fwd", "train", "train")), dtype, N, C, max(1, min(L, most // (N * C))), G,
                     rng.choice(("none", "relu", "silu", "silu")), rng.random() < 0.4, ragged)
    C = _log_int(rng, 1, 512)
    L = max(1, min(L, most // (N * C)))
    if op == "dropout":
        return _dropout("", dtype, N, C, L, rng.choice((0.1, 0.2, 0.5, 0.05)), rng.random() < 0.7, ragged)
    use = rng.choice(("fwd", "train", "train", "step"))
    return _embed("", use, dtype, N, C, 1 if use == "step" else L, _log_int(rng, 2, 32000), rng.choice((1.0, C ** 0.5)), rng.random() < 0.7,
                  ragged and use != "step")


def draw(rng):
    c = _draw(rng)
    del c["name"]
    return c


# ---- inputs -----------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    t = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    N, L, train = case["N"], case["L"], case["use"] == "train"
    st = {"case": case, "lengths": None}
    if case["ragged"]:
        lengths = (L * torch.rand(N, generator=gen, device=dev)).ceil().to(torch.int32).clamp(0, L)
        lengths[0] = L
        st["lengths"] = lengths
    if case["op"] == "embed":
        V, D = case["V"], case["D"]
        # the k-th most frequent token is met 1 / k times as often as the first; which number a token has says nothing of that
        rank = (torch.exp(torch.rand(N, L, generator=gen, device=dev, dtype=torch.float64) * math.log(V + 1.0)) - 1).long().clamp(0, V - 1)
        tokens = torch.randperm(V, generator=gen, device=dev)[rank].to(torch.int64 if case["wide"] else torch.int32)
        st["tokens"] = tokens[:, 0].contiguous() if case["use"] == "step" else tokens
        st["table"] = normal(V, D).to(t)
        st["dy"] = normal(N, D, L).to(t) if train else None
        return st
    C = case["C"]
    if case["op"] == "dropout":
        st.update(x=normal(N, C, L).to(t), residual=normal(N, C, L).to(t) if case["residual"] else None, dy=normal(N, C, L).to(t))
        # the generator's key and the number of the call
        st["key"], st["call"] = (int(v) for v in torch.randint(0, 2 ** 62, (2,), generator=gen, device=dev).tolist())
        return st

    def activations(at, spread):
        if case["last"]:
            return (at + spread * normal(N, L, C)).to(t).transpose(1, 2)
        return (torch.as_tensor(at, device=dev)[..., None] + torch.as_tensor(spread, device=dev)[..., None] * normal(N, C, L)).to(t)

    # what a layer leaves: every channel with a mean and a spread of its own
    st["x"] = activations(0.5 * normal(C), 0.5 + torch.rand(C, generator=gen, device=dev))
    st["dy"] = activations(0, 1) if train else None
    st["weight"], st["bias"] = 1 + 0.1 * normal(C), 0.1 * normal(C)
    return st


# ---- one pass ---------------------------------------------------------------------------------------------------------
def run(state):
    if own:
        return _own(state)
    return {"embed": _plain_embed, "norm": _plain_norm, "dropout": _plain_dropout}[state["case"]["op"]](state)


def _own(st):
    from paper_2104_08002_amd import blocks

    case = st["case"]
    if case["op"] == "embed":
        if case["use"] == "step":
            return blocks.conv1d_embed_step(st["table"], st["tokens"], scale=case["scale"])
        y = blocks.conv1d_embed_fwd(st["table"], st["tokens"], scale=case["scale"], lengths=st["lengths"])
        if case["use"] == "fwd":
            return y
        return y, blocks.conv1d_embed_bwd(st["dy"], st["tokens"], case["V"], scale=case["scale"], lengths=st["lengths"])
    if case["op"] == "dropout":
        y = blocks.conv1d_dropout(st["x"], case["p"], st["key"], st["call"], residual=st["residual"], lengths=st["lengths"])
        return y, blocks.conv1d_dropout(st["dy"], case["p"], st["key"], st["call"], lengths=st["lengths"])
    how = {"weight": st["weight"], "bias": st["bias"], "relu": case["act"] == "relu", "silu": case["act"] == "silu", "lengths": st["lengths"]}
    if case["use"] == "fwd":
        return blocks.conv1d_norm_fwd(st["x"], case["G"], **how)
    y, stats = blocks.conv1d_norm_fwd(st["x"], case["G"], **how, want_stats=True)
    dx, dweight, dbias = blocks.conv1d_norm_bwd(st["dy"], stats, st["x"], case["G"], **how)
    return y, dx, dweight, dbias


def _inside(st, L):
    """True where a position lies within its sequence, [N, 1, L]; None where all do."""
    if st["lengths"] is None:
        return None
    return (torch.arange(L, device="cuda") < st["lengths"][:, None])[:, None]


def _plain_embed(st):
    case, t = st["case"], st["table"].dtype
    V, D, tokens = case["V"], case["D"], st["tokens"].long()
    if case["use"] == "step":
        return (case["scale"] * st["table"].float()[tokens]).to(t)
    inside = _inside(st, case["L"])
    y = (case["scale"] * st["table"].float()[tokens]).to(t).transpose(1, 2)
    y = y.contiguous() if inside is None else torch.where(inside, y, 0.0)
    if case["use"] == "fwd":
        return y
    dy = st["dy"] if inside is None else torch.where(inside, st["dy"], 0.0)
    # sums up to and with each position in the order of the tokens, taken at the ends of their runs
    of, order = torch.sort(tokens.view(-1), stable=True)
    upto = torch.nn.functional.pad(dy.transpose(0, 1).reshape(D, -1)[:, order].double().cumsum(1), (1, 0))
    v = torch.arange(V, device="cuda")
    dtable = upto[:, torch.searchsorted(of, v, right=True)] - upto[:, torch.searchsorted(of, v)]
    return y, (case["scale"] * dtable.T).float().contiguous()


def _plain_norm(st):
    case, x = st["case"], st["x"].float()
    N, C, L = x.shape
    G, t = case["G"], st["x"].dtype
    inside = _inside(st, L)
    if inside is not None:
        x = torch.where(inside, x, 0.0)
    count = torch.full((N,), L, device="cuda") if inside is None else st["lengths"].clamp(min=1)
    count = (C // G * count.double()).view(N, 1, 1, 1)

    def whole(v):
        """Sums over a group's channels and positions."""
        return v.view(N, G, -1, L).sum((2, 3), keepdim=True, dtype=torch.float64)

    x = x.contiguous().view(N, G, -1, L)
    mean = whole(x) / count
    off = x.double() - mean
    if inside is not None:
        off = torch.where(inside[:, None], off, 0.0)
    rstd = torch.rsqrt(whole(off * off) / count + 1e-5)
    # (in 64 bits up to here: which side of 0 a value lies on decides over its gradient)
    h = (off * rstd).view(N, C, L)
    positive = h * st["weight"].double()[:, None] + st["bias"].double()[:, None] > 0
    h, rstd = h.float(), rstd.float()
    w, b = st["weight"][:, None], st["bias"][:, None]
    p = h * w + b
    if case["act"] == "silu":
        s = torch.sigmoid(p)
        y, slope = p * s, s * (1 + p * (1 - s))
    elif case["act"] == "relu":
        y, slope = p.clamp(min=0), positive.float()
    else:
        y, slope = p, torch.ones_like(p)
    if inside is not None:
        y = torch.where(inside, y, 0.0)

    def as_input(v):
        return v.to(t).transpose(1, 2).contiguous().transpose(1, 2) if case["last"] else v.to(t)

    if case["use"] == "fwd":
        return as_input(y)
    dp = st["dy"].float() * slope
    if inside is not None:
        dp = torch.where(inside, dp, 0.0)
    g = dp * w
    first, second = ((whole(v.contiguous()) / count).float().expand(N, G, C // G, 1).reshape(N, C, 1) for v in (g, g * h))
    dx = rstd.expand(N, G, C // G, 1).reshape(N, C, 1) * (g - first - h * second)
    if inside is not None:
        dx = torch.where(inside, dx, 0.0)
    return as_input(y), as_input(dx), (dp * h).sum((0, 2), dtype=torch.float64).float(), dp.sum((0, 2), dtype=torch.float64).float()


_M = 0xffffffff


def _words(rows, L, key, call):
    """Word (row, l) of Philox4x32 in seven rounds: counter row * ceil(L / 4) + l / 4 and `call`, key `key`, word l % 4."""
    blocks = rows * ((L + 3) // 4)
    at = torch.arange(blocks, device="cuda")
    c = [at & _M, at >> 32, torch.full_like(at, call & _M), torch.full_like(at, call >> 32 & _M)]
    k0, k1 = key & _M, key >> 32 & _M
    for _ in range(7):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32 & _M) ^ c[1] ^ k0, b & _M, (a >> 32 & _M) ^ c[3] ^ k1, a & _M]
        k0, k1 = (k0 + 0x9E3779B9) & _M, (k1 + 0xBB67AE85) & _M
    return torch.stack(c, 1).view(rows, -1)[:, :L]


def _plain_dropout(st):
    case, x = st["case"], st["x"]
    N, C, L = x.shape
    kept = (_words(N * C, L, st["key"], st["call"]) >= math.floor(case["p"] * 2.0 ** 32)).view(N, C, L)
    inside = _inside(st, L)
    if inside is not None:
        kept = kept & inside
    scale = 1 / (1 - case["p"])
    y, dx = torch.where(kept, x.float() * scale, 0.0), torch.where(kept, st["dy"].float() * scale, 0.0)
    if st["residual"] is not None:
        y = y + (st["residual"].float() if inside is None else torch.where(inside, st["residual"].float(), 0.0))
    return y.to(x.dtype), dx.to(x.dtype)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    N, L = case["N"], case["L"]
    if case["op"] == "embed":
        e, V, D = N * L * case["D"], case["V"], case["D"]
        fwd = size * (e + min(V, N * L) * D) + N * L * (8 if case["wide"] else 4)
        if case["use"] == "train":
            return {"bytes": fwd + size * e + 4 * V * D, "flops": 3 * e}
        return {"bytes": fwd, "flops": e}
    e = N * L * case["C"]
    if case["op"] == "dropout":
        # (two 32-bit products and six other operations a round, of which four elements have seven)
        return {"bytes": size * (4 + int(case["residual"])) * e, "flops": 2 * (16 + 2) * e}
    act = {"none": 0, "relu": 1, "silu": 5}[case["act"]]
    if case["use"] == "train":
        return {"bytes": size * 4 * e, "flops": (24 + 3 * act) * e}
    return {"bytes": size * 2 * e, "flops": (7 + act) * e}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    return {"embed": _exact_embed, "norm": _exact_norm, "dropout": _exact_dropout}[case["op"]](st)


def _exact_embed(st):
    case, table = st["case"], st["table"].double()
    if case["use"] == "step":
        return table[st["tokens"].long()] * case["scale"]
    N, D, L, V = case["N"], case["D"], case["L"], case["V"]
    lengths = [L] * N if st["lengths"] is None else st["lengths"].tolist()
    y = torch.zeros(N, D, L, dtype=torch.float64, device="cuda")
    seen, rows = [], []
    for n, m in enumerate(lengths):
        of = st["tokens"][n, :m].long()
        y[n, :, :m] = table[of].T * case["scale"]
        if case["use"] == "train":
            seen.append(of)
            rows.append(st["dy"][n, :, :m].T.double())
    if case["use"] != "train":
        return y
    # a product with the truth values "this row has that token", some tokens at a time
    of, rows = torch.cat(seen)[:, None], torch.cat(rows)
    some = max(1, 2 ** 27 // max(1, len(rows)))
    parts = [(of == torch.arange(v, min(V, v + some), device="cuda")).double().T.contiguous() @ rows for v in range(0, V, some)]
    return y, case["scale"] * torch.cat(parts)


def _exact_norm(st):
    case = st["case"]
    N, C, L, G = case["N"], case["C"], case["L"], case["G"]
    lengths = [L] * N if st["lengths"] is None else st["lengths"].tolist()
    train, per = case["use"] == "train", C // G
    y, dx = (torch.zeros(N, C, L, dtype=torch.float64, device="cuda") for _ in range(2))
    dw, db = (torch.zeros(C, dtype=torch.float64, device="cuda") for _ in range(2))
    for n, m in enumerate(lengths):
        if m == 0:
            continue
        for g in range(G):
            of = slice(g * per, (g + 1) * per)
            x, w, b = st["x"][n, of, :m].double(), st["weight"][of, None].double(), st["bias"][of, None].double()
            mean = x.mean()
            root = (((x - mean) ** 2).mean() + 1e-5).sqrt()
            h = (x - mean) / root
            p = w * h + b
            sig = 1 / (1 + torch.exp(-p))
            y[n, of, :m] = {"none": p, "relu": torch.where(p > 0, p, 0.0), "silu": p * sig}[case["act"]]
            if not train:
                continue
            dp = st["dy"][n, of, :m].double()
            if case["act"] == "silu":
                dp = dp * (sig + p * sig * (1 - sig))
            elif case["act"] == "relu":
                dp = torch.where(p > 0, dp, 0.0)
            dw[of] += (dp * h).sum(1)
            db[of] += dp.sum(1)
            dh = dp * w
            dx[n, of, :m] = (dh - dh.mean() - h * (dh * h).mean()) / root
    return (y, dx, dw, db) if train else y


def _exact_dropout(st):
    case = st["case"]
    N, C, L = st["x"].shape
    key, call, per = st["key"], st["call"], -(-L // 4)
    # the generator again, its products of 32 bits from halves of 16, one word of a block after the other
    low = lambda v: v % 65536  # noqa: E731

    def product(v, m):
        m0, m1 = m % 65536, m // 65536
        mid = low(v) * m1 + low(v) * m0 // 65536
        mid, carry = (v // 65536) * m0 + mid % 65536, mid // 65536
        return (v // 65536) * m1 + carry + mid // 65536, (mid % 65536) * 65536 + (low(v) * m0) % 65536

    at = torch.arange(N * C * per, device="cuda")
    x0, x1 = at % 2 ** 32, at // 2 ** 32
    x2, x3 = torch.full_like(at, call % 2 ** 32), torch.full_like(at, call // 2 ** 32)
    for turn in range(7):
        hi0, lo0 = product(x0, 0xD2511F53)
        hi2, lo2 = product(x2, 0xCD9E8D57)
        x0, x1, x2, x3 = (hi2 ^ x1 ^ (key + turn * 0x9E3779B9) % 2 ** 32, lo2, hi0 ^ x3 ^ (key // 2 ** 32 + turn * 0xBB67AE85) % 2 ** 32, lo0)
    words = torch.stack((x0, x1, x2, x3), 1).reshape(N * C, 4 * per)[:, :L].reshape(N, C, L)
    kept = words.double() / 2.0 ** 32 >= math.floor(case["p"] * 2.0 ** 32) / 2.0 ** 32
    if st["lengths"] is not None:
        behind = torch.arange(L, device="cuda")[None, None] >= st["lengths"][:, None, None]
    else:
        behind = torch.zeros(1, 1, L, dtype=torch.bool, device="cuda")
    y, dx = (torch.where(kept, v.double() / (1 - case["p"]), 0.0) for v in (st["x"], st["dy"]))
    if st["residual"] is not None:
        y = y + st["residual"].double()
    return y.masked_fill(behind, 0.0), dx.masked_fill(behind, 0.0)
